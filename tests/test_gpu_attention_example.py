"""The example runs, and what it serves from 8 bits is what 16 bits give, as far as 8 bits tell."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_example():
    from paper_2404_04541_amd import attention_example as ex
    from paper_2404_04541_amd import binding as sg
    torch.manual_seed(1)
    handle = sg.Handle()
    pattern = ex.two_step_pattern(handle, 16)
    assert pattern.rows == pattern.cols == 16 and pattern.nnz > 16
    o, grads = ex.training_step(handle)
    assert torch.isfinite(o).all() and all(torch.isfinite(g).all() and g.abs().max() > 0 for g in grads)
    out, want, live = ex.serve(handle)
    assert live == 5      # 130 tokens twice: three pages each, the first of them (whole when the row was forked) shared
    # keys and values are off by at most 2^-4 each (three bits and a half after the point): a tenth in the mean square is generous
    assert float((out.float() - want.float()).norm() / want.float().norm()) < 0.1
