"""RetentionStep.return_freed: what a redirect freed goes back once, whoever calls it how often; captured too."""
import pytest

import synth
from paper_2606_09916_amd.step import RetentionStep
from test_gpu_slots import Stack
from test_gpu_turn_e2m1 import _batch

pytestmark = pytest.mark.gpu


def _freed(st):
    return [u for b in range(2) for u in st.freed[st.sess[b].slot_off:st.sess[b].slot_off + int(st.n_freed[b])].tolist()]


def test_once_only(dev):
    st = RetentionStep(_batch(64, synth.F32, 84), dev)
    st.init_dead_slot()
    stack = Stack([], st.num_slots, dev)
    st.return_freed(stack.free)
    assert stack() == []                                 # before the first event
    st.step()
    gone = _freed(st)
    assert len(gone) > 100
    for _ in range(2):
        st.return_freed(stack.free)
        assert stack() == gone and st.n_freed.tolist() == [0, 0]
    st.redirect()                                        # the positions are dropped already
    st.return_freed(stack.free)
    assert stack() == gone
    # an event that is taken back
    st.reset()
    st.step()
    assert _freed(st) == gone
    st.reset()
    other = Stack([], st.num_slots, dev)
    st.return_freed(other.free)
    assert other() == []


def test_captured_with_the_event(dev):
    import torch
    st = RetentionStep(_batch(64, synth.F32, 85), dev)
    st.init_dead_slot()
    st.step()
    gone = _freed(st)
    stack = Stack([], st.num_slots, dev)

    def turn():
        st.redirect()
        st.return_freed(stack.free)

    st.reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        turn()
    torch.cuda.current_stream().wait_stream(side)
    assert stack() == gone
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for _ in range(3):
        stack.count.zero_()
        st.reset()
        graph.replay()
        torch.cuda.synchronize()
        assert stack() == gone and st.n_freed.tolist() == [0, 0]
        st.return_freed(stack.free)                      # once more, eagerly
        graph.replay()                                   # and an event with nothing left to free
        assert stack() == gone
