"""Pieces of a window with attention nodes, captured: each replay computes its frames from the frames before them."""
import pytest

from oracle import graph_oracle as go
from tests.test_gpu_layer_nodes import compare, long_workload, window_of

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def window(T):
    w = long_workload(T, 2, False)
    win = window_of(w, T)
    win.forward()
    win.bptt()
    win.compute_grads()      # everything is loaded
    torch.cuda.synchronize()
    ref = go.forward_bptt(w.spec.nodes, w.spec.edges, w.weights, w.biases, w.inputs, w.targets, T, 2)

    def right(label):
        win.bptt()
        win.compute_grads()
        torch.cuda.synchronize()
        compare(win, ref, w.spec, label)
    return win, right


def capture(work):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    return graph


@pytest.mark.parametrize("T,a,b", [(24, 8, 16), (90, 70, 85), (90, 3, 88)])
def test_a_piece_replayed(T, a, b):
    win, right = window(T)
    win.forward_range(0, a)
    piece = capture(lambda: win.forward_range(a, b))
    for _ in range(3):
        piece.replay()
    win.forward_range(b, T)
    right("replayed piece")
    # the same frames again, and pieces that run at once in front of and behind replays
    win.forward_range(0, a)
    win.forward_range(a, b)
    piece.replay()
    win.forward_range(b, T)
    piece.replay()
    win.forward_range(a, T)
    right("piece between others")


def test_two_pieces_in_one_capture_and_a_whole_window_between_pieces():
    T = 40
    win, right = window(T)
    win.forward_range(0, 10)
    both = capture(lambda: (win.forward_range(10, 20), win.forward_range(20, T)))
    for _ in range(3):
        both.replay()
        right("two pieces")
    whole = capture(lambda: win.forward())
    win.forward_range(0, 10)
    whole.replay()
    win.forward_range(10, 25)
    whole.replay()
    win.forward_range(25, T)
    right("pieces between whole windows")
