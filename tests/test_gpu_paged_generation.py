"""The paged calls together, as a program uses them (examples/paged_generation.py)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import __graft_entry__ as g
    g.build()
    from examples import paged_generation
    return paged_generation


@pytest.mark.parametrize("native", [False, True], ids=["e4m3", "native"])
def test_drafts_change_nothing_but_the_passes(example, native):
    """The most likely tokens are the same with drafts and without, in fewer passes."""
    one = example.generate(drafts=0, tokens=24, native=native, greedy=True)
    many = example.generate(drafts=4, tokens=24, native=native, greedy=True)
    assert one[0] == many[0]
    assert one[1] == 24 and many[1] < 24


def test_answer_becomes_a_chunk(example):
    answer, passes, chunk = example.generate(drafts=3, tokens=20)
    assert len(answer) == 20 and all(0 <= t < example.VOCAB for t in answer)
    assert chunk["n_slots"] == -(-chunk["n_tokens"] // example.RATIO) and chunk["n_tokens"] >= 19
