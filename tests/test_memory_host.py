"""What a memory refuses before it touches a GPU."""
import pytest

from paper_2303_04670_amd import evconv as ev


@pytest.mark.parametrize("bad", [dict(recall_pages=0), dict(recall_pages=1), dict(recall_pages=-3), dict(recall_pages=65537), dict(recall_windows=0), dict(recall_windows=-64),
                                 dict(longest=0), dict(heads_v=3, heads_k=2), dict(heads_v=0), dict(heads_k=0), dict(recall=(2,)), dict(recall=(-1, 0)),
                                 dict(recall_windows=1 << 30), dict(recall_windows=1 << 30, recall_pages=3)])
def test_layers_that_look_back_are_refused_when_they_are_made(bad):
    """Not by the first window, behind the layers that have rewritten their states by then."""
    pytest.importorskip("torch")
    from paper_2303_04670_amd.memory import Memory
    with pytest.raises(ev.EvConvError) as e:
        Memory(**{**dict(dim=96, n_streams=4, n_out=11, recall=(0, 1), device="cpu"), **bad})
    assert "expected a GPU" not in str(e.value)  # (what its weights' first call would say)
