"""Networks with norm, attention and dropout nodes on the GPU, against the float64 graph oracle."""
import numpy as np
import pytest

import workloads as wl
from oracle import graph_oracle as go
from tests.test_gpu_parity import GRAD_TOL, OUT_TOL, nerr, run_both
from tests.test_layer_nodes import small_net

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T, N", [(1, 1), (2, 3), (5, 1), (19, 2), (70, 5)])
@pytest.mark.parametrize("gain", [True, False])
def test_every_connection_kind(T, N, gain):
    run_both(wl.make_workload("layers", small_net(np.random.default_rng(0), gain), T, N, seed=T, scale=0.8), label=f"layers T={T} N={N} gain={gain}")


@pytest.mark.parametrize("T, N, dim, heads", [(1, 2, 32, 2), (3, 1, 64, 1), (33, 3, 48, 3), (64, 2, 40, 5), (131, 2, 96, 1), (9, 2, 300, 2), (600, 1, 32, 2)])
def test_attention_net(T, N, dim, heads):
    """600 frames of one stream and two heads are cut into segments; 300 units: heads of 150, columns in two slices."""
    w = wl.make_workload("attention", wl.attention_net(11, dim, heads, 2, 7, dropout=0.25), T, N, seed=4, scale=0.25)
    run_both(w, label=f"attention T={T} N={N} {heads} x {dim // heads}")


def test_framewise_norm_and_dropout(monkeypatch):
    monkeypatch.setenv("RNNG_SCHEDULE", "framewise")
    g = wl.GraphSpec()
    x = g.add_node(wl.INPUT, wl.LINEAR, 5, name="x")
    h = wl.add_lstm_layer(g, x, 24, "L")["h"]
    n = g.add_node(wl.NORM, wl.LINEAR, 24, has_bias=True, name="norm")
    g.add_edge(h, n, wl.IDENTITY)
    g.add_edge(x, n, wl.FULL, 1)
    d = g.add_node(wl.DROPOUT, wl.LINEAR, 24, name="drop", dropout=(0.5, 3, 0))
    g.add_edge(n, d, wl.IDENTITY, 2)
    out = g.add_node(wl.ADD, wl.SOFTMAX, 6, has_bias=True, is_output=1, name="out")
    g.add_edge(d, out, wl.FULL)
    g.add_edge(n, out, wl.FULL)
    run_both(wl.make_workload("framewise", g, 13, 3, seed=2), label="framewise")


def long_workload(total, N, delayed, seed=5):
    spec = small_net(np.random.default_rng(1)) if delayed else wl.attention_net(11, 48, 3, 1, 7, dropout=0.25)
    return wl.make_workload("long", spec, total, N, seed=seed, scale=0.4)


def window_of(w, T):
    """A window over the first T frames of workload w."""
    from paper_1503_02852_amd.runner import window_for
    return window_for(wl.Workload("window", w.spec, T, w.N, w.weights, w.biases, {k: v[:T] for k, v in w.inputs.items()}, {k: v[:T] for k, v in w.targets.items()}))


def compare(win, ref, spec, label):
    for k, n in enumerate(spec.nodes):
        if n["kind"] == wl.INPUT:
            continue
        assert nerr(win.node_output(k), ref["y"][k]) < OUT_TOL, (label, n["name"])
        assert nerr(win.node_state_grad(k), -ref["delta"][k]) < GRAD_TOL, (label, "ds", n["name"])
    gw, gb = win.grads_unpacked()
    for a, b in zip(gw + gb, ref["grad_w"] + ref["grad_b"]):
        if b is not None:
            assert nerr(a, b) < GRAD_TOL, (label, "gradient")


@pytest.mark.parametrize("delayed", [False, True])
@pytest.mark.parametrize("T, steps", [(12, (6, 6, 6)), (80, (3, 70, 40, 1))])
def test_window_moved_ahead(T, steps, delayed):
    """Outputs and gradients of every window; the state in front of it is what all earlier frames left."""
    w = long_workload(T + sum(steps), 2, delayed)
    n, e = w.spec.nodes, w.spec.edges
    y, z = go.forward(n, e, w.weights, w.biases, w.inputs, T + sum(steps), w.N)
    win = window_of(w, T)
    win.forward()
    first = 0
    for step in (0,) + steps:
        if step:
            cut = slice(first + T, first + T + step)
            win.advance({k: v[cut] for k, v in w.inputs.items()}, {k: v[cut] for k, v in w.targets.items()})
            first += step
        win.bptt()
        win.compute_grads()
        compare(win, go.bptt_window(n, e, w.weights, w.biases, y, z, w.targets, first, T, w.N), w.spec, f"window at {first}")


def test_window_in_pieces():
    """Pieces of any length, one of them computed twice (its earlier frames are there)."""
    w = long_workload(100, 3, False)
    win = window_of(w, 100)
    for t0, t1 in ((0, 1), (1, 40), (40, 90), (33, 35), (35, 100)):
        win.forward_range(t0, t1)
    win.bptt()
    win.compute_grads()
    compare(win, go.forward_bptt(w.spec.nodes, w.spec.edges, w.weights, w.biases, w.inputs, w.targets, 100, 3), w.spec, "pieces")


def test_captured_window_moves_on_in_every_replay():
    import torch
    T, step, N = 24, 8, 2
    w = long_workload(T + 5 * step, N, False)
    n, e = w.spec.nodes, w.spec.edges
    y, z = go.forward(n, e, w.weights, w.biases, w.inputs, T + 5 * step, N)
    win = window_of(w, T)
    xs = {k: torch.from_numpy(v).to(win.dev) for k, v in w.inputs.items()}
    ts = {k: torch.from_numpy(v).to(win.dev).to(win.targets[k].dtype) for k, v in w.targets.items()}

    def move(first):
        for k, v in xs.items():
            win.inputs[k].copy_(v[first:first + T])
        for k, v in ts.items():
            win.targets[k].copy_(v[first:first + T])

    def work():
        win.g.shift_window(step, win._stream())
        win.forward_range(T - step, T)
        win.bptt()
        win.compute_grads()

    win.forward()
    win.bptt()
    win.compute_grads()
    move(step)
    work()                                   # eager: everything is loaded
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(2, 6):
        move(i * step)
        graph.replay()
        torch.cuda.synchronize()
        compare(win, go.bptt_window(n, e, w.weights, w.biases, y, z, w.targets, i * step, T, N), w.spec, f"replay {i}")


def test_captured_training_step_draws_anew():
    """A fresh window captured with a device offset: each replay's gradients are the oracle's with that offset."""
    import torch
    w = long_workload(20, 2, False)
    win = window_of(w, 20)
    off = torch.zeros(1, dtype=torch.int64, device=win.dev)
    for k, n in enumerate(w.spec.nodes):
        if n["kind"] == wl.DROPOUT:
            p, seed, offset = n["dropout"]
            win.g.set_dropout(k, p, seed, offset, off.data_ptr())
    (out,) = w.spec.output_nodes()
    y = torch.empty(20, 2, w.spec.nodes[out]["dim"], device=win.dev)

    def work():
        win.g.forward_static(win.weights.data_ptr(), win._input_ptrs(), [y.data_ptr()], 20, 2, win._stream())
        win.bptt()
        win.compute_grads()

    win.step()
    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in (0, 1, 5, 1):
        off.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        nodes = [dict(n, dropout=(n["dropout"][0], n["dropout"][1], n["dropout"][2] + i)) if "dropout" in n else n for n in w.spec.nodes]
        ref = go.forward_bptt(nodes, w.spec.edges, w.weights, w.biases, w.inputs, w.targets, 20, 2)
        gw, gb = win.grads_unpacked()
        for a, b in zip(gw + gb, ref["grad_w"] + ref["grad_b"]):
            if b is not None:
                assert nerr(a, b) < GRAD_TOL, i


def test_static_workspace():
    import torch
    w = long_workload(40, 2, False)
    win = window_of(w, 40)
    win.forward()
    ref, _ = go.forward(w.spec.nodes, w.spec.edges, w.weights, w.biases, w.inputs, 40, 2)
    out = w.spec.output_nodes()[0]
    y = torch.empty(40, 2, w.spec.nodes[out]["dim"], device=win.dev)
    win.g.forward_static(win.weights.data_ptr(), win._input_ptrs(), [y.data_ptr()], 40, 2, win._stream())
    torch.cuda.synchronize()
    assert nerr(y.cpu().numpy(), ref[out]) < OUT_TOL


def test_deterministic_bits():
    w = long_workload(150, 3, False)
    win = window_of(w, 150)
    win.g.set_deterministic()
    seen = []
    for _ in range(3):
        win.step()
        seen.append(win.grads.cpu().numpy().copy())
    assert np.array_equal(seen[0], seen[1]) and np.array_equal(seen[0], seen[2])


def test_setters_end_the_window():
    from paper_1503_02852_amd import RnnError
    w = long_workload(12, 1, False)
    win = window_of(w, 12)
    drop = next(k for k, n in enumerate(w.spec.nodes) if n["kind"] == wl.DROPOUT)
    att = next(k for k, n in enumerate(w.spec.nodes) if n["kind"] == wl.ATTENTION)
    win.forward()
    win.g.set_dropout(drop, 0.0, 1)
    with pytest.raises(RnnError, match="before rnn_forward"):
        win.bptt()
    win.forward()
    win.g.set_attention(att, 3, win.log_decay[att].data_ptr())
    with pytest.raises(RnnError, match="computed window"):
        win.g.shift_window(1)
    with pytest.raises(RnnError, match="have not been computed"):
        win.forward_range(6, 12)
    win.forward()
    ref, _ = go.forward([dict(n, scale=1.0, **({"dropout": (0.0, 0, 0)} if k == drop else {})) for k, n in enumerate(w.spec.nodes)], w.spec.edges, w.weights, w.biases, w.inputs, 12, 1)
    out = w.spec.output_nodes()[0]
    assert nerr(win.node_output(out), ref[out]) < OUT_TOL


def test_character_model():
    """The configuration with its own widths and one-hot input given as class indices, over a shorter window."""
    w = wl.make_config("charlm_attention_n32", T=70, N=4, bias_scale=0.1)
    run_both(w, check_all_nodes=False, label=w.name)
    win = window_of(w, 70)
    win.set_onehot_inputs({k: v.argmax(-1) for k, v in w.inputs.items()})
    win.step()
    ref = go.forward_bptt(w.spec.nodes, w.spec.edges, w.weights, w.biases, w.inputs, w.targets, 70, 4)
    gw, gb = win.grads_unpacked()
    for a, b in zip(gw + gb, ref["grad_w"] + ref["grad_b"]):
        if b is not None:
            assert nerr(a, b) < GRAD_TOL


def test_class_indices_straight_into_the_layers():
    """One-hot inputs given as class indices whose connections lead into norm and attention nodes, one of them delayed."""
    g = wl.GraphSpec()
    x = g.add_node(wl.INPUT, wl.LINEAR, 9, name="x")
    n = g.add_node(wl.NORM, wl.LINEAR, 32, has_bias=True, name="norm")
    g.add_edge(x, n, wl.FULL)
    g.add_edge(x, n, wl.FULL, 2)
    a = g.add_node(wl.ATTENTION, wl.LINEAR, 32, name="att", heads=2, scale=0.3, log_decay=np.array([-0.05, -0.5]))
    g.add_edge(x, a, wl.FULL)
    g.add_edge(n, a, wl.IDENTITY)
    g.add_edge(x, a, wl.FULL, 1)
    out = g.add_node(wl.ADD, wl.SOFTMAX, 5, has_bias=True, is_output=1, name="out")
    g.add_edge(a, out, wl.FULL)
    g.add_edge(n, out, wl.FULL)
    T, N = 37, 3
    w = wl.make_workload("classes", g, T, N, seed=6, scale=0.5)
    idx = np.random.default_rng(8).integers(-1, 9, size=(T, N))
    w.inputs[x] = np.where(idx[..., None] >= 0, np.eye(9, dtype=np.float32)[idx], 0).astype(np.float32)
    win = window_of(w, T)
    win.set_onehot_inputs({x: idx})
    win.step()
    compare(win, go.forward_bptt(g.nodes, g.edges, w.weights, w.biases, w.inputs, w.targets, T, N), g, "classes")


def test_layers_between_recurrent_layers():
    """LSTM -> norm -> LSTM -> attention: the recurrent layers run as their step kernels, the layers between their launches."""
    g = wl.GraphSpec()
    x = g.add_node(wl.INPUT, wl.LINEAR, 12, name="x")
    h = wl.add_lstm_layer(g, x, 32, "L1")["h"]
    n = g.add_node(wl.NORM, wl.LINEAR, 32, has_bias=True, name="norm")
    g.add_edge(h, n, wl.IDENTITY)
    d = g.add_node(wl.DROPOUT, wl.LINEAR, 32, name="drop", dropout=(0.2, 11, 3))
    g.add_edge(n, d, wl.IDENTITY)
    h2 = wl.add_lstm_layer(g, d, 32, "L2")["h"]
    a = g.add_node(wl.ATTENTION, wl.LINEAR, 32, name="att", heads=4, scale=0.35, log_decay=-np.array([0.0, 0.1, 0.01, 1.0]))
    for _ in range(3):
        g.add_edge(h2, a, wl.FULL)
    out = g.add_node(wl.ADD, wl.SOFTMAX, 5, has_bias=True, is_output=1, name="out")
    g.add_edge(a, out, wl.FULL)
    g.add_edge(h2, out, wl.FULL)
    for N in (1, 20):
        run_both(wl.make_workload("stack", g, 50, N, seed=N, scale=0.3), label=f"stack N={N}")


def test_layers_read_in_place():
    """Layers on a lone identity connection: of an input, of another layer, of a recurrent layer; all three of attention's from one node.  The
    window moves on, so that the copies of inputs and the layers' tensors are shifted."""
    g = wl.GraphSpec()
    x = g.add_node(wl.INPUT, wl.LINEAR, 24, name="x")
    n = g.add_node(wl.NORM, wl.LINEAR, 24, name="norm")
    g.add_edge(x, n, wl.IDENTITY)
    d = g.add_node(wl.DROPOUT, wl.LINEAR, 24, name="drop", dropout=(0.4, 2, 0))
    g.add_edge(n, d, wl.IDENTITY)
    a = g.add_node(wl.ATTENTION, wl.LINEAR, 24, name="att", heads=3, scale=0.3, log_decay=np.array([-0.3, -0.02, 0.0]))
    for _ in range(3):
        g.add_edge(d, a, wl.IDENTITY)
    h = wl.add_lstm_layer(g, a, 24, "L")["h"]
    n2 = g.add_node(wl.NORM, wl.LINEAR, 24, has_bias=True, name="norm2")
    g.add_edge(h, n2, wl.IDENTITY)
    out = g.add_node(wl.ADD, wl.SOFTMAX, 5, has_bias=True, is_output=1, name="out")
    g.add_edge(n2, out, wl.FULL)
    g.add_edge(n, out, wl.FULL, 3)
    T, step, N = 20, 7, 3
    w = wl.make_workload("in place", g, T + 2 * step, N, seed=12, scale=0.3)
    y, z = go.forward(g.nodes, g.edges, w.weights, w.biases, w.inputs, T + 2 * step, N)
    win = window_of(w, T)
    win.forward()
    for i in range(3):
        if i:
            cut = slice(T + (i - 1) * step, T + i * step)
            win.advance({k: v[cut] for k, v in w.inputs.items()}, {k: v[cut] for k, v in w.targets.items()})
        win.bptt()
        win.compute_grads()
        compare(win, go.bptt_window(g.nodes, g.edges, w.weights, w.biases, y, z, w.targets, i * step, T, N), g, f"in place {i}")
