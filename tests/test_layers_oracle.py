"""Pins of the layers' oracle: its gradients against differences of its own forward pass, linear attention against
the sum over pairs of frames, the dropout generator against published values."""
import numpy as np
import pytest

from oracle import layers_oracle as lo


def case(seed, T=5, N=3, H=4, Hk=2, dk=3, dv=2):
    r = np.random.default_rng(seed)
    g = lambda *s: r.standard_normal(s)  # noqa: E731
    x = dict(q=g(T, N, H, dk), k=g(T, N, Hk, dk), v=g(T, N, Hk, dv), state=g(N, H, dk, dv))
    return x, np.array([-0.3, 0.0, -np.inf, -2.0])[:H], np.array([T, 2, 0])[:N], g(T, N, H, dv), g(N, H, dk, dv)


def test_attention_is_the_decayed_sum_over_pairs():
    x, a, L, _, _ = case(1)
    o, S = lo.attention_forward(**{n: x[n] for n in "qkv"}, log_decay=a, scale=0.7, state=x["state"], lengths=L)
    for n in range(3):
        for h in range(4):
            for t in range(5):
                want = np.zeros(2)
                if t < L[n]:
                    want = 0.7 * np.exp(a[h] * (t + 1)) * x["q"][t, n, h] @ x["state"][n, h]
                    for s in range(t + 1):
                        w = 1.0 if s == t else np.exp(a[h] * (t - s))
                        want = want + 0.7 * w * (x["q"][t, n, h] @ x["k"][s, n, h // 2]) * x["v"][s, n, h // 2]
                assert np.allclose(o[t, n, h], want, rtol=1e-12, atol=1e-13)
    assert np.array_equal(S[2], x["state"][2])


@pytest.mark.parametrize("name", ["q", "k", "v", "state"])
def test_attention_gradients_against_differences(name):
    x, a, L, do, dS = case(2)

    def error(y):
        o, S = lo.attention_forward(y["q"], y["k"], y["v"], a, 0.7, y["state"], L)
        return (o * do).sum() + (S * dS).sum()

    grads = dict(zip(("q", "k", "v", "state"), lo.attention_backward(x["q"], x["k"], x["v"], a, 0.7, do, x["state"], dS, L)))
    step = 1e-4
    for at in np.ndindex(x[name].shape):
        up, down = ({n: y.copy() for n, y in x.items()} for _ in range(2))
        up[name][at] += step
        down[name][at] -= step
        # the error is a polynomial, linear in each of q, k, v and state: the central difference is exact but for rounding
        assert abs((error(up) - error(down)) / (2 * step) - grads[name][at]) < 1e-9


def test_generator_gives_the_published_values():
    ones, pi = 0xFFFFFFFF, (0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344)
    # test vectors that the generator's authors publish
    for rounds, ctr, key, want in [(10, (0, 0, 0, 0), (0, 0), "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
                                   (10, (ones,) * 4, (ones, ones), "408f276d 41c83b0e a20bc7c6 6d5451fd"),
                                   (10, pi, (0xA4093822, 0x299F31D0), "d16cfe09 94fdcceb 5001e420 24126ea1"),
                                   (7, (0, 0, 0, 0), (0, 0), "5f6fb709 0d893f64 4f121f81 4f730a48")]:
        got = lo.philox4x32(np.array(ctr, np.uint32), key, rounds)
        assert " ".join(f"{w:08x}" for w in got) == want


def test_dropout_keeps_the_share_it_should():
    f = lo.dropout_factor(2000, 1001, 0.3, (5 << 32) + 9, (7 << 33) + 1)
    kept = (f > 0).mean()
    assert abs(kept - 0.7) < 5 * np.sqrt(0.21 / f.size)      # five standard deviations
    assert np.isclose(f.max(), 1 / 0.7, rtol=2.0 ** -16)
    assert np.array_equal(f[5:9], lo.dropout_factor(4, 1001, 0.3, (5 << 32) + 9, (7 << 33) + 1, first_row=5))


@pytest.mark.parametrize("name", ["x", "residual", "gain"])
def test_add_norm_gradients_against_differences(name):
    r = np.random.default_rng(3)
    x = dict(x=r.standard_normal((3, 7)), residual=r.standard_normal((3, 7)), gain=r.standard_normal(7))
    dy, dh = r.standard_normal((3, 7)), r.standard_normal((3, 7))
    factor = lo.dropout_factor(3, 7, 0.4, 11, 0)

    def error(y):
        h, out, _ = lo.add_norm(y["x"], y["residual"], y["gain"], 1e-3, factor)
        return (out * dy).sum() + (h * dh).sum()

    h, _, rstd = lo.add_norm(x["x"], x["residual"], x["gain"], 1e-3, factor)
    dx, dres, dgain = lo.add_norm_backward(dy, dh, h, rstd, x["gain"], factor)
    grad = {"x": dx, "residual": dres, "gain": dgain}[name]
    step = 1e-5
    for at in np.ndindex(x[name].shape):
        up, down = ({n: y.copy() for n, y in x.items()} for _ in range(2))
        up[name][at] += step
        down[name][at] -= step
        # third derivatives of order 10, step^2 = 1e-10, rounding 1e-16 / step
        assert abs((error(up) - error(down)) / (2 * step) - grad[at]) < 1e-8
