"""Linear attention: what bf16 inputs may cost.  The inputs and the stored results are bf16, everything between them counts in 32 bits, however
the terms of a result cancel and whatever else the call is asked for.

u = 2^-24.  A result is a sum of terms of which `mag` is the sum of absolute values (the oracle with absolute inputs).  A term passes, at
worst, a rounding for every addition of a product over dk and dv (twice as many where one factor comes in two bf16 numbers), for every frame of a
chunk in a product over frames (three times for the state's update, in three numbers), three for every frame between (decay, its own error, the
product), H / Hk for shared heads and a few more: each takes at most u of the partial sum, which is at most mag.  A score, or the state as an operand of
an output, in two bf16 numbers is off by 2^-16 = 256 u of itself at most; a term passes one of the two."""
import numpy as np
import pytest

from tests.test_gpu_layers import CASES, DEV, U, Attention, half_step, host

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def roundings(c):
    T, N, H, Hk, dk, dv = c.shape
    return 8 * T + 4 * (dk + dv) + H // Hk + 64 + (256 if c.t == torch.bfloat16 else 0)


class Exact(Attention):
    def tolerance(self, mag, stored, want):
        return U * roundings(self) * mag + half_step(stored) * np.abs(want) + 1e-37

    def set(self, name, values):
        """Frames inside the streams' lengths."""
        T, N = self.shape[:2]
        values = torch.from_numpy(np.broadcast_to(values, self.x[name].shape).astype(np.float32)).to(DEV).to(self.t)
        for n in range(N):
            last = T if self.lengths_host is None else min(max(self.lengths_host[n], 0), T)
            self.x[name][:last, n] = values[:last, n]

    def check_norms(self, names, backward):
        """Roundings of one result are independent of each other, each uniform within u (a third of its square on average) of a partial sum of at most about
        the result's own size, for a typical one: u (roundings / 3)^(1/2) of the results' norm, three times that at most; and what stores them."""
        want = self.oracle(False, backward)
        for name in names:
            stored = self.t if name in self.x else torch.float32
            e = np.linalg.norm(host(self.x[name] if name in self.x else getattr(self, name)) - want[name]) / np.linalg.norm(want[name])
            rest = half_step(stored) * (1 / 3) ** 0.5 if stored == torch.bfloat16 else 0.0
            assert e <= 3 * U * ((3 * self.shape[0] + 32) / 3) ** 0.5 + rest, (name, e)


def run_and_check(c):
    c.forward()
    c.check(("o", "state_out"), False)
    c.backward()
    c.check(("dq", "dk", "dv", "dstate"), True)


@pytest.mark.parametrize("T,N,H,Hk,dk,dv,lengths", CASES)
def test_every_size_within_32_bits(T, N, H, Hk, dk, dv, lengths):
    print(f"[attention] {T} {N} {H} {Hk} {dk} {dv} {lengths}", flush=True)
    run_and_check(Exact(T, N, H, Hk, dk, dv, "bf16", lengths, seed=T + dv))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", [(16, 64), (150, 64), (150, 128), (70, 256), (600, 32)])
@pytest.mark.parametrize("kind", ["offset", "alternating"])
def test_terms_that_cancel(kind, T, d, dtype):
    """Keys and values around one with queries (and gradients of the outputs) that sum up to nothing: what the keys and values share
    drops out of each product with the state.  Equal keys with values of alternating sign: two frames drop out against each other."""
    c = Exact(T, 1, 2, 1, d, d, dtype, seed=T, decays=[-0.001, -0.02])
    r = np.random.default_rng(d)
    normal = lambda *s: r.standard_normal(s)  # noqa: E731
    if kind == "offset":
        for name in ("k", "v"):
            c.set(name, 1 + 0.2 * normal(T, 1, 1, d))
        for name in ("q", "do"):
            x = normal(T, 1, 2, d)
            c.set(name, x - x.mean(-1, keepdims=True))
    else:
        c.set("k", normal(1, 1, 1, d))
        c.set("v", normal(1, 1, 1, d) * (-1.0) ** np.arange(T)[:, None, None, None])
        c.set("q", normal(1, 1, 2, d))
    run_and_check(c)


@pytest.mark.parametrize("T", [16, 64, 150, 300])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_states_keep_24_bits(T, dtype):
    """An update that came in 16 bits would take 2^-17 / 3^(1/2) of the state's norm, 4.4e-6; the bound is 1.3e-6 for 150 frames."""
    c = Exact(T, 1, 4, 4, 128, 128, dtype, seed=T, decays=[0.0, -0.002, -0.01, -0.1])
    c.forward()
    c.backward()
    c.check_norms(("o", "state_out"), False)
    c.check_norms(("dq", "dk", "dv", "dstate"), True)


@pytest.mark.parametrize("T", [20, 64, 200])
def test_the_same_bits_whatever_else_is_asked_for(T):
    """Outputs with and without the last state, gradients with and without the state's, all of them in one segment."""
    c = Exact(T, 1, 2, 1, 64, 64, "bf16", seed=3)
    x = c.x
    c.forward()
    c.backward()
    o = torch.full_like(x["o"], c.MARK)
    c.layer.forward(x["q"], x["k"], x["v"], c.log_decay, o, state=c.state)
    assert torch.equal(o, x["o"])
    with_state = {n: torch.full_like(x[n], c.MARK) for n in ("dq", "dk", "dv")}
    c.layer.backward(x["q"], x["k"], x["v"], c.log_decay, x["do"], **with_state, state=c.state, dstate_out=c.dstate_out)
    assert all(torch.equal(with_state[n], x[n]) for n in with_state)
    for n in with_state:
        alone = torch.full_like(x[n], c.MARK)
        c.layer.backward(x["q"], x["k"], x["v"], c.log_decay, x["do"], **{n: alone}, state=c.state, dstate_out=c.dstate_out)
        assert torch.equal(alone, x[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_chunks_and_single_frames_agree(dtype):
    """A window at once and in calls of at most three frames, keys and values around one: the state handed on either way, within both bounds."""
    from paper_1503_02852_amd import layers
    T, d = 130, 64
    c = Exact(T, 1, 2, 1, d, d, dtype, seed=1, decays=[-0.001, 0.0])
    r = np.random.default_rng(1)
    for name in ("k", "v"):
        c.set(name, 1 + 0.2 * r.standard_normal((T, 1, 1, d)))
    q = r.standard_normal((T, 1, 2, d))
    c.set("q", q - q.mean(-1, keepdims=True))
    c.forward()
    c.check(("o", "state_out"), False)
    state, o, at = c.state.clone(), torch.empty_like(c.x["o"]), 0
    while at < T:
        n = min(1 + at % 3, T - at)
        piece = layers.LinearAttention(n, 1, 2, d, d, kv_heads=1, dtype=c.t, scale=c.scale, device=DEV)
        cut = lambda a: a[at:at + n]  # noqa: E731
        piece.forward(cut(c.x["q"]), cut(c.x["k"]), cut(c.x["v"]), c.log_decay, cut(o), state=state, state_out=state)
        at += n
    mag, want = c.oracle(True), c.oracle()
    assert (np.abs(host(o) - host(c.x["o"])) <= 2 * c.tolerance(mag["o"], c.t, want["o"])).all()
    assert (np.abs(host(state) - host(c.state_out)) <= 2 * c.tolerance(mag["state_out"], torch.float32, want["state_out"])).all()
    c.x["o"], c.state_out = o, state
    c.check(("o", "state_out"), False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(1, 1), (3, 40), (40, 3), (7, 7), (2, 200), (130, 5)])
@pytest.mark.parametrize("T,layout", [(5, "frames"), (70, "heads"), (150, "streams"), (1000, "frames")])
def test_heads_of_less_than_16_bytes(T, layout, dk, dv, dtype):
    run_and_check(Exact(T, 2, 4, 2, dk, dv, dtype, [T, T - 3], seed=T + dk, layout=layout))


@pytest.mark.parametrize("dk,dv", [(3, 3), (16, 16)])
def test_decays_next_to_one_over_many_frames(dk, dv):
    """exp(-1e-7) has no neighbour in fp32 nearer than 1.9e-8, which 20,000 frames would make 3.8e-4 of what the first state leaves; bound: 2.6e-5."""
    c = Exact(20000, 1, 2, 2, dk, dv, "f32", seed=1, decays=[-1e-7, -3e-7])
    c.state *= 1000
    c.dstate_out *= 1000
    c.forward()
    c.check_norms(("o", "state_out"), False)
    c.backward()
    c.check_norms(("dq", "dk", "dv", "dstate"), True)
