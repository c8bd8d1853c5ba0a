"""The example of serving with drafted tokens runs, and its texts and cache stay in step."""
import pytest

pytestmark = pytest.mark.gpu


def test_serving_with_drafts():
    from paper_2404_04541_amd import binding as sg
    from paper_2404_04541_amd import draft_example
    text, rate = draft_example.serve(sg.Handle(), steps=8)
    assert [len(t) > p for t, p in zip(text, (40, 7, 130))] == [True] * 3
    assert 1 <= rate <= 4 and all(0 <= x < 300 for t in text for x in t)
