"""Norm, attention and dropout nodes: the oracle against differences and the layers' own oracle; the library's graph rules."""
import numpy as np
import pytest

import workloads as wl
from oracle import graph_oracle as go
from oracle import layers_oracle as lo
from paper_1503_02852_amd import Graph, RnnError


def small_net(rng, gain=True):
    """Every connection kind and a delay into each kind of node, an LSTM layer in front."""
    g = wl.GraphSpec()
    x = g.add_node(wl.INPUT, wl.LINEAR, 3, name="x")
    h = wl.add_lstm_layer(g, x, 4, "L")["h"]
    n = g.add_node(wl.NORM, wl.LINEAR, 4, has_bias=gain, name="norm")
    g.add_edge(x, n, wl.FULL, 2)
    g.add_edge(h, n, wl.IDENTITY)
    g.add_edge(h, n, wl.DIAG, 1)
    a = g.add_node(wl.ATTENTION, wl.LINEAR, 4, name="att", heads=2, scale=0.7, log_decay=np.array([-0.1, -1.5]))
    g.add_edge(n, a, wl.FULL)
    g.add_edge(h, a, wl.DIAG, 1)
    g.add_edge(n, a, wl.IDENTITY)
    d = g.add_node(wl.DROPOUT, wl.LINEAR, 4, name="drop", dropout=(0.3, 5, 9))
    g.add_edge(a, d, wl.FULL)
    g.add_edge(n, d, wl.IDENTITY, 1)
    m = g.add_node(wl.MUL, wl.TANH, 4, name="mul")
    g.add_edge(d, m, wl.IDENTITY)
    g.add_edge(a, m, wl.IDENTITY)
    out = g.add_node(wl.ADD, wl.SOFTMAX, 3, has_bias=True, is_output=1, name="out")
    g.add_edge(m, out, wl.FULL)
    g.add_edge(d, out, wl.FULL, 1)
    return g


@pytest.mark.parametrize("gain", [True, False])
def test_oracle_gradients_by_differences(gain):
    rng = np.random.default_rng(0)
    w = wl.make_workload("layers", small_net(rng, gain), 5, 2, seed=3, scale=0.8)
    n, e = w.spec.nodes, w.spec.edges
    W = [None if x is None else x.astype(np.float64) for x in w.weights]
    B = [None if x is None else x.astype(np.float64) for x in w.biases]
    ref = go.forward_bptt(n, e, W, B, w.inputs, w.targets, w.T, w.N)
    E = lambda: go.loss(n, go.forward(n, e, W, B, w.inputs, w.T, w.N)[0], w.targets)  # noqa: E731
    for p, g in zip(W + B, ref["grad_w"] + ref["grad_b"]):
        if p is None:
            continue
        for i in np.ndindex(p.shape):
            keep = p[i]
            p[i] = keep + 1e-5
            up = E()
            p[i] = keep - 1e-5
            down = E()
            p[i] = keep
            assert abs((up - down) / 2e-5 - g[i]) < 1e-7 * max(1.0, abs(g[i]))      # h^2 f''' / 6 and 2^-53 E / h: both below 1e-9


def test_oracle_window_gradient_holds_the_state_constant():
    """bptt_window's gradient of frames [3, 7): differences of the window's error with everything before it held fixed."""
    g = wl.GraphSpec()
    x = g.add_node(wl.INPUT, wl.LINEAR, 4, name="x")
    a = g.add_node(wl.ATTENTION, wl.LINEAR, 4, name="att", heads=2, scale=1.0, log_decay=np.array([-0.2, 0.0]))
    for _ in range(3):
        g.add_edge(x, a, wl.FULL)
    out = g.add_node(wl.ADD, wl.SOFTMAX, 3, is_output=1, name="out")
    g.add_edge(a, out, wl.FULL)
    w = wl.make_workload("window", g, 7, 2, seed=1, scale=0.8)
    n, e = g.nodes, g.edges
    W = [x.astype(np.float64) for x in w.weights]
    y, z = go.forward(n, e, W, w.biases, w.inputs, 7, 2)
    ref = go.bptt_window(n, e, W, w.biases, y, z, w.targets, 3, 4, 2)
    xs = w.inputs[0].astype(np.float64)
    proj = lambda m, t0, t1, V: (xs[t0:t1] @ V[m].T).reshape(t1 - t0, 2, 2, 2)  # noqa: E731
    _, S = lo.attention_forward(*(proj(m, 0, 3, W) for m in range(3)), n[1]["log_decay"], 1.0)

    def E(V):
        o, _ = lo.attention_forward(*(proj(m, 3, 7, V) for m in range(3)), n[1]["log_decay"], 1.0, state=S)
        s = o.reshape(4, 2, 4) @ V[3].T
        p = s - np.log(np.exp(s).sum(-1, keepdims=True))
        return -np.take_along_axis(p, w.targets[2][3:, :, None].astype(int), -1).sum()

    assert abs(E(W) - ref["loss"]) < 1e-12
    for m in range(4):
        for i in np.ndindex(W[m].shape):
            V = [v.copy() for v in W]
            V[m][i] += 1e-5
            up = E(V)
            V[m][i] -= 2e-5
            assert abs((up - E(V)) / 2e-5 - ref["grad_w"][m][i]) < 1e-7


X, O = [wl.INPUT, 0, 4, 0, 0], [wl.ADD, wl.SOFTMAX, 3, 0, 1]


@pytest.mark.parametrize("nodes, edges, word", [
    ([X, [4, wl.TANH, 4, 1, 0], O], [[0, 1, 0, 0], [1, 2, 0, 0]], "no activation"),
    ([X, [5, 0, 4, 1, 0], O], [[0, 1, 0, 0]] * 3 + [[1, 2, 0, 0]], "no bias"),
    ([X, [6, 0, 4, 1, 0], O], [[0, 1, 0, 0], [1, 2, 0, 0]], "no bias"),
    ([X, [4, 0, 16385, 1, 0], O], [[0, 1, 0, 0], [1, 2, 0, 0]], "16384"),
    ([X, [5, 0, 4, 0, 0], O], [[0, 1, 0, 0]] * 2 + [[1, 2, 0, 0]], "three incoming"),
    ([X, [5, 0, 4, 0, 0], O], [[0, 1, 0, 0]] * 4 + [[1, 2, 0, 0]], "three incoming"),
    ([X, [4, 0, 4, 0, 0], O], [[1, 2, 0, 0]], "without incoming"),
    ([X, [4, 0, 4, 0, 1]], [[0, 1, 0, 0]], "softmax"),
    ([X, [6, 0, 4, 0, 2]], [[0, 1, 0, 0]], "squared-error"),
    ([X, [4, 0, 4, 0, 0], O], [[0, 1, 0, 0], [1, 1, 1, 2], [1, 2, 0, 0]], "recurrent"),
    ([X, [6, 0, 4, 0, 0], [wl.ADD, wl.TANH, 4, 0, 0], O], [[0, 1, 0, 0], [1, 2, 0, 0], [2, 1, 1, 0], [2, 3, 0, 0]], "recurrent"),
])
def test_graph_rules(nodes, edges, word):
    with pytest.raises(RnnError, match=word):
        Graph(nodes, edges)


def test_setters_refuse():
    g = Graph([X, [5, 0, 6, 0, 0], [6, 0, 6, 0, 0], O], [[0, 1, 0, 0]] * 3 + [[1, 2, 0, 2], [2, 3, 0, 0]])
    for T, N in ((5, 2), (1, 1)):
        with pytest.raises(RnnError, match="rnn_set_attention"):
            g.workspace_bytes(T, N)
    d = 1 << 20      # (an address: nothing runs)
    for node, heads, scale, ptr, word in ((2, 2, 1.0, d, "attention node"), (0, 1, 1.0, d, "attention node"), (9, 1, 1.0, d, "attention node"), (1, 0, 1.0, d, "heads"),
                                          (1, 4, 1.0, d, "heads"), (1, 2, float("nan"), d, "scale"), (1, 2, float("inf"), d, "scale"),
                                          (1, 2, 1.0, 0, "log_decay"), (1, 2, 1.0, d + 1, "log_decay")):
        with pytest.raises(RnnError, match=word):
            g.set_attention(node, heads, ptr, scale)
    for node, p, ptr, word in ((1, 0.5, None, "dropout node"), (-1, 0.5, None, "dropout node"), (2, -0.1, None, "probability"), (2, 1.5, None, "probability"),
                               (2, float("nan"), None, "probability"), (2, 0.5, d + 4, "aligned")):
        with pytest.raises(RnnError, match=word):
            g.set_dropout(node, p, 1, 0, ptr)
    g.set_attention(1, 2, d)
    two = g.workspace_bytes(64, 300)
    g.set_attention(1, 6, d)
    assert g.workspace_bytes(64, 300) < two      # 6 heads of 1 x 1 instead of 2 of 3 x 3
    g.set_dropout(2, 0.5, 1)
    with pytest.raises(RnnError, match="2\\^20"):
        g.workspace_bytes(4, 1 << 18)
    wide = Graph([X, [5, 0, 512, 0, 0], O], [[0, 1, 0, 0]] * 3 + [[1, 2, 0, 0]])
    with pytest.raises(RnnError, match="256"):
        wide.set_attention(1, 1, d)
    wide.set_attention(1, 2, d)


def test_framewise_schedule_is_refused(monkeypatch):
    monkeypatch.setenv("RNNG_SCHEDULE", "framewise")
    with pytest.raises(RnnError, match="framewise"):
        Graph([X, [5, 0, 4, 0, 0], O], [[0, 1, 0, 0]] * 3 + [[1, 2, 0, 0]])
    Graph([X, [4, 0, 4, 0, 0], O], [[0, 1, 0, 0], [1, 2, 0, 0]])


def test_workspace_of_a_part_fits_the_window():
    """A part of a window may be cut into as many segments as the whole: its workspace is never larger."""
    import ctypes
    from paper_1503_02852_amd import load_library
    from paper_1503_02852_amd.binding import LinearAttentionDesc
    lib = load_library()
    for heads, d in ((1, 64), (3, 128), (37, 32), (8, 200)):
        last = 0
        for T in list(range(1, 700)) + list(range(700, 40000, 997)):
            b = lib.rnn_linear_attention_workspace_bytes(ctypes.byref(LinearAttentionDesc(T, 1, heads, heads, d, d, 0, 1.0)), 0)
            assert b >= last
            last = b


def test_no_streams_in_a_long_window():
    import ctypes
    from paper_1503_02852_amd import load_library
    from paper_1503_02852_amd.binding import LinearAttentionDesc
    for T in (0, 1, 5, 1000):
        for backward in (0, 1):
            assert load_library().rnn_linear_attention_workspace_bytes(ctypes.byref(LinearAttentionDesc(T, 0, 4, 2, 16, 16, 1, 1.0)), backward) == 0
