"""Cases of the layers that need no step loop: linear attention with a decay for each head, the residual sum with
dropout and root-mean-square norm, and dropout by itself.

With `own` false, `run` computes them in elementary torch operations (32 bits, rounded once at the end); with `own`
true it makes the calls of paper_1503_02852_amd.layers that a user's program makes.

Layouts are the library's: frames x streams x heads x units, [T][N][heads][dim], and rows x units for the row layers.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda:0"
EPS = 1e-6


def _attention(name, op, dtype, T, N, heads, kv_heads, dk, dv, ragged=False, carry=True):
    c = dict(kind="attention", op=op, dtype=dtype, T=T, N=N, heads=heads, kv_heads=kv_heads, dk=dk, dv=dv, ragged=ragged, carry=carry)
    return dict(c, name=name) if name else c


def _norm(name, op, dtype, rows, dim, residual=True, p=0.0, group=0):
    c = dict(kind="norm", op=op, dtype=dtype, rows=rows, dim=dim, residual=residual, p=p, group=group)
    return dict(c, name=name) if name else c


def _dropout(name, dtype, rows, dim, p):
    c = dict(kind="dropout", dtype=dtype, rows=rows, dim=dim, p=p)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one running sequence, one new frame of a character model: the smallest serving call
        _attention("step_n1", "forward", "bf16", 1, 1, 8, 8, 64, 64),
        # one new frame of 192 running sequences, four query heads to a key head: the state is what is read and written
        _attention("step_n192", "forward", "bf16", 1, 192, 16, 4, 128, 128),
        # a prompt of one sequence, its state handed on to the single frames that follow
        _attention("prompt_n1", "forward", "bf16", 4096, 1, 16, 16, 128, 128),
        # a training window of eight streams, forward and backward, state carried in, gradient of the state carried out
        _attention("train_n8", "train", "bf16", 2048, 8, 16, 16, 128, 128),
        # streams of several lengths (some empty, some of one frame), shared key heads, sizes that fill no tile, in the graphs' own type
        _attention("train_ragged", "train", "f32", 777, 5, 6, 2, 40, 56, ragged=True),
        # one very long sequence: work split along time
        _attention("long_n1", "forward", "bf16", 65536, 1, 8, 2, 128, 128),
        # one new frame: launch latency
        _norm("norm_step", "forward", "f32", 1, 512),
        # a training window's residual sum with dropout and norm, and the way back
        _norm("norm_forward", "forward", "bf16", 8192, 4096, p=0.1),
        _norm("norm_backward", "backward", "bf16", 8192, 4096, p=0.1),
        # the norm in front of products in 8 bits: a scale for each 128 units
        _norm("norm_e4m3", "e4m3", "bf16", 16384, 4096, group=128),
        # between the layers of the 32-stream character model, there and back
        _dropout("dropout_n32", "f32", 8192, 512, 0.25),
        # the largest: a word model's width, rows that fill no vector
        _dropout("dropout_odd", "bf16", 4099, 16381, 0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "norm", "dropout"])
    if kind == "attention":
        op = rng.choice(["step", "forward", "train"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        kv_heads = _log_int(rng, 1, 16)
        heads = kv_heads * rng.choice([1, 1, 2, 4])
        dk = rng.choice([64, 128, _log_int(rng, 16, 256)])
        dv = rng.choice([dk, dk, _log_int(rng, 16, 256)])
        if op == "step":
            N = _log_int(rng, 1, max(1, min(256, (192 * 16 * 128 * 128) // (heads * dk * dv))))
            return _attention(None, "forward", dtype, rng.choice([1, 1, 2, 5]), N, heads, kv_heads, dk, dv)
        most = (5 if op == "train" else 10) * 10 ** 6 // (heads * max(dk, dv))      # frames of all streams together
        N = _log_int(rng, 1, min(32, most // 32))
        T = _log_int(rng, 17, max(18, min(65536 if op == "forward" else 8192, most // N)))
        return _attention(None, op, dtype, T, N, heads, kv_heads, dk, dv, ragged=rng.random() < 0.4, carry=rng.random() < 0.6)
    dtype = rng.choice(["bf16", "f16", "f32"])
    rows, dim = _log_int(rng, 1, 32768), _log_int(rng, 32, 16384)
    if rng.random() < 0.6:
        dim = max(32, dim // 32 * 32)
    rows = max(1, min(rows, (32 << 20) // dim))
    if kind == "dropout":
        return _dropout(None, dtype, rows, dim, round(rng.uniform(0.05, 0.7), 3))
    op = rng.choice(["forward", "backward", "e4m3"])
    return _norm(None, op, dtype, rows, dim, residual=rng.random() < 0.7, p=rng.choice([0.0, 0.1, 0.3]), group=rng.choice([0, 128]) if op == "e4m3" else 0)


def work(case):
    c, b = case, SIZE[case["dtype"]]
    if c["kind"] == "attention":
        frames = c["T"] * c["N"] * (0.5 if c["ragged"] else 1.0)
        q, k = frames * c["heads"] * c["dk"], frames * c["kv_heads"] * c["dk"]
        o, v = frames * c["heads"] * c["dv"], frames * c["kv_heads"] * c["dv"]
        state = c["N"] * c["heads"] * c["dk"] * c["dv"]
        products = frames * c["heads"] * c["dk"] * c["dv"]
        n_states = 2 if c["carry"] else 1
        if c["op"] == "forward":
            return {"bytes": (q + k + v + o) * b + n_states * state * 4, "flops": 4 * products}
        return {"bytes": (q + k + v + o) * b + (2 * (q + k + v) + o) * b + (2 * n_states + 1) * state * 4, "flops": 14 * products}
    n = c["rows"] * c["dim"]
    if c["kind"] == "dropout":
        return {"bytes": 4 * n * b, "flops": 2 * n}
    if c["op"] == "backward":      # dy, the gradient of the sum, the sum; gradients of the layer's input and of the residual
        writes = 2 if c["residual"] and c["p"] > 0 else 1
        return {"bytes": (3 + writes) * n * b, "flops": 8 * n}
    reads = 2 if c["residual"] else 1
    if c["op"] == "e4m3":
        return {"bytes": (reads + 1) * n * b + n + c["rows"] * 4 * (c["dim"] // 128 if c["group"] else 1), "flops": 8 * n}
    return {"bytes": (reads + 2) * n * b, "flops": 6 * n}


class _State(dict):
    __getattr__ = dict.__getitem__


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    host = np.random.RandomState(seed % (1 << 31))
    t = TYPES[case["dtype"]]

    def gauss(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)

    def empty(*shape, dtype=t):
        return torch.zeros(*shape, device=DEV, dtype=dtype)

    s = _State(case=case)
    if case["kind"] == "attention":
        T, N, H, Hk, dk, dv = (case[n] for n in ("T", "N", "heads", "kv_heads", "dk", "dv"))
        s["q"], s["k"], s["v"] = gauss(T, N, H, dk), gauss(T, N, Hk, dk, scale=0.5), gauss(T, N, Hk, dv)
        # time constants from a few frames to thousands; one head in eight forgets nothing
        rates = np.exp2(-host.uniform(1.5, 11.0, H))
        rates[host.uniform(size=H) < 0.125] = 0.0
        s["log_decay"] = torch.from_numpy(np.log1p(-rates).astype(np.float32)).to(DEV)
        s["scale"] = 1.0 / math.sqrt(dk)
        lengths = np.full(N, T)
        if case["ragged"]:
            lengths = host.randint(0, T + 1, N)
            lengths[host.randint(N)] = T
            if N > 2:
                lengths[np.argsort(lengths)[:2]] = (0, 1)
        s["lengths_host"] = lengths
        s["lengths"] = torch.from_numpy(lengths.astype(np.int32)).to(DEV) if case["ragged"] else None
        s["state"] = gauss(N, H, dk, dv, dtype=torch.float32) if case["carry"] else None
        s["o"], s["state_out"] = empty(T, N, H, dv), empty(N, H, dk, dv, dtype=torch.float32)
        if case["op"] == "train":
            s["do"] = gauss(T, N, H, dv)
            s["dstate_out"] = gauss(N, H, dk, dv, dtype=torch.float32) if case["carry"] else None
            s["dq"], s["dk"], s["dv"] = empty(T, N, H, dk), empty(T, N, Hk, dk), empty(T, N, Hk, dv)
            s["dstate"] = empty(N, H, dk, dv, dtype=torch.float32)
        if own:
            from paper_1503_02852_amd import layers
            s["layer"] = layers.LinearAttention(T, N, H, dk, dv, kv_heads=Hk, dtype=t, scale=s.scale, training=case["op"] == "train", device=DEV)
        return s
    rows, dim = case["rows"], case["dim"]
    s["seed"], s["offset"] = int(host.randint(1 << 30)) * 4294967311 % (1 << 63), int(host.randint(1 << 30))
    if case["kind"] == "dropout":
        s["x"], s["dy"] = gauss(rows, dim), gauss(rows, dim)
        s["y"], s["dx"] = empty(rows, dim), empty(rows, dim)
        return s
    s["gain"] = 1.0 + gauss(dim, scale=0.2, dtype=torch.float32)
    if own:
        from paper_1503_02852_amd import layers
        s["layer"] = layers.AddNorm(rows, dim, dtype=t, eps=EPS, dropout=case["p"], seed=s.seed, offset=s.offset, device=DEV)
    if case["op"] == "backward":
        s["dy"], s["h"], s["dh"] = gauss(rows, dim), gauss(rows, dim, scale=2.0), gauss(rows, dim)
        s["rstd"] = (s.h.double().square().mean(1) + EPS).rsqrt().float()
        s["dx"], s["dgain"] = empty(rows, dim), empty(dim, dtype=torch.float32)
        s["dresidual"] = empty(rows, dim) if case["residual"] and case["p"] > 0 else None
        return s
    s["x"] = gauss(rows, dim)
    s["residual"] = gauss(rows, dim, scale=2.0) if case["residual"] else None
    s["h"] = empty(rows, dim)
    if case["op"] == "e4m3":
        s["y"], s["scales"] = empty(rows, dim, dtype=torch.float8_e4m3fn), empty(rows, -(-dim // 128) if case["group"] else 1, dtype=torch.float32)
    else:
        s["y"], s["rstd"] = empty(rows, dim), empty(rows, dtype=torch.float32)
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------
def _powers(log_decay, n):
    """exp(log_decay n) for every head and every number in n (angles in 64 bits), [heads][...]."""
    a = log_decay.double().view(-1, *([1] * n.dim()))
    return torch.exp(a * n.double()).float()


def _past(q, k, v, log_decay, C=128):
    """sum over j <= i of decay^(i - j) (q_i . k_j) v_j, [N][H][T][.], in chunks of C frames."""
    N, H, T, dk = q.shape
    dv = v.shape[-1]
    nc = -(-T // C)
    cut = lambda x: torch.nn.functional.pad(x, (0, 0, 0, nc * C - T)).view(N, H, nc, C, x.shape[-1])  # noqa: E731
    q, k, v = cut(q), cut(k), cut(v)
    i = torch.arange(C, device=q.device)
    lag = i[:, None] - i[None, :]
    near = _powers(log_decay, lag.clamp(min=0)) * (lag >= 0)
    out = torch.matmul(torch.matmul(q, k.transpose(-1, -2).contiguous()) * near[:, None], v)
    if nc > 1:
        sums = torch.matmul((k * _powers(log_decay, C - 1 - i)[:, None, :, None]).transpose(-1, -2).contiguous(), v)
        c = torch.arange(nc, device=q.device)
        gap = c[:, None] - c[None, :] - 1
        before = torch.matmul((_powers(log_decay, gap.clamp(min=0) * C) * (gap >= 0))[None], sums.view(N, H, nc, dk * dv)).view(N, H, nc, dk, dv)
        out = out + torch.matmul(q, before) * _powers(log_decay, i + 1)[:, None, :, None]
    return out.reshape(N, H, nc * C, dv)[:, :, :T]


def _heads_first(x, heads=None):
    x = x.float().permute(1, 2, 0, 3)
    return x if heads is None or x.shape[1] == heads else x.repeat_interleave(heads // x.shape[1], 1)


def _frames_first(x, kv_heads, like):
    N, H, T, d = x.shape
    return x.view(N, kv_heads, H // kv_heads, T, d).sum(2).permute(2, 0, 1, 3).to(like.dtype).contiguous()


def _plain_attention(s):
    c = s.case
    H, T, a = c["heads"], c["T"], s.log_decay
    q, k, v = _heads_first(s.q), _heads_first(s.k, H), _heads_first(s.v, H)
    t = torch.arange(T, device=q.device)
    if s.lengths is None:
        L, there = torch.full((c["N"],), T, device=q.device), None
        left = _powers(a, T - 1 - t)[None, :, :, None]
    else:
        L = s.lengths.long()
        there = (t[None, :] < L[:, None]).float()[:, None, :, None]
        q, k, v = q * there, k * there, v * there
        left = _powers(a, (L[:, None] - 1 - t).clamp(min=0)).permute(1, 0, 2)[..., None] * there
    whole = _powers(a, L).permute(1, 0)[:, :, None, None]
    since = _powers(a, t + 1)[None, :, :, None]
    o = _past(q, k, v, a)
    state = torch.matmul((k * left).transpose(-1, -2).contiguous(), v)
    if s.state is not None:
        o = o + torch.matmul(q, s.state) * since
        state = state + whole * s.state
    out = {"o": _frames_first(o * s.scale, H, s.o), "state": state}
    if c["op"] == "forward":
        return out
    do = _heads_first(s.do)
    do = do if there is None else do * there
    dq = _past(do, v, k, a)
    dk = _past(v.flip(2), do.flip(2), q.flip(2), a).flip(2) * s.scale
    dv = _past(k.flip(2), q.flip(2), do.flip(2), a).flip(2) * s.scale
    dstate = torch.matmul((q * since).transpose(-1, -2).contiguous(), do) * s.scale
    if s.state is not None:
        dq = dq + torch.matmul(do, s.state.transpose(-1, -2).contiguous()) * since
        dk = dk + torch.matmul(v, s.dstate_out.transpose(-1, -2).contiguous()) * left
        dv = dv + torch.matmul(k, s.dstate_out) * left
        dstate = dstate + whole * s.dstate_out
    out.update(dq=_frames_first(dq * s.scale, H, s.dq), dk=_frames_first(dk, c["kv_heads"], s.dk), dv=_frames_first(dv, c["kv_heads"], s.dv), dstate=dstate)
    return out


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def _plain_keep(rows, dim, p, seed, offset):
    """Which elements dropout keeps, [rows][dim]: Philox4x32 of seven rounds (Salmon, Moraes, Dror and Shaw, 2011), eight 16-bit
    numbers of one counter for eight neighbouring units."""
    groups = -(-dim // 8)
    low = 0xFFFFFFFF
    n = torch.arange(rows * groups, device=DEV, dtype=torch.int64)
    c = [n & low, n >> 32, torch.full_like(n, offset & low), torch.full_like(n, offset >> 32)]
    key = [seed & low, seed >> 32]

    def product(m, x):      # high and low word of m x
        lo = m * (x & 0xFFFF)
        hi = m * (x >> 16) + (lo >> 16)
        return hi >> 16, ((hi & 0xFFFF) << 16) | (lo & 0xFFFF)

    for _ in range(7):
        h0, l0 = product(0xD2511F53, c[0])
        h1, l1 = product(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    words = torch.stack(c, 1)
    u = torch.stack([words & 0xFFFF, words >> 16], 2).view(rows, groups * 8)[:, :dim]
    return u >= _threshold(p)


def _plain_dropped(x, p, seed, offset):
    x = x.float()
    if _threshold(p) == 0:
        return x
    keep = _plain_keep(x.shape[0], x.shape[1], p, seed, offset)
    return torch.where(keep, x * (65536.0 / (65536 - _threshold(p))), torch.zeros_like(x))


def _plain_norm(s):
    c = s.case
    if c["op"] == "backward":
        dy, n = s.dy.float(), s.h.float() * s.rstd[:, None]
        g = dy * s.gain
        dh = s.dh.float() + s.rstd[:, None] * (g - n * (g * n).mean(1, keepdim=True))
        out = {"dx": _plain_dropped(dh, c["p"], s.seed, s.offset).to(s.dx.dtype), "dgain": (dy * n).sum(0)}
        if s.dresidual is not None:
            out["dresidual"] = dh.to(s.dx.dtype)
        return out
    h = _plain_dropped(s.x, c["p"], s.seed, s.offset)
    if s.residual is not None:
        h = h + s.residual.float()
    rstd = torch.rsqrt(h.square().mean(1) + EPS)
    y = h * rstd[:, None] * s.gain
    out = {"h": h.to(s.x.dtype)}
    if c["op"] == "forward":
        out.update(y=y.to(s.x.dtype), rstd=rstd)
        return out
    rows, dim = y.shape
    width = 128 if c["group"] else dim
    blocks = -(-dim // width)
    y = torch.nn.functional.pad(y, (0, blocks * width - dim)).view(rows, blocks, width)
    scales = y.abs().amax(2) / 448.0
    scales = torch.where(scales > 0, scales, torch.ones_like(scales))
    y = (y / scales[..., None]).clamp(-448.0, 448.0).view(rows, blocks * width)[:, :dim]
    out.update(y=y.to(torch.float8_e4m3fn), scales=scales)
    return out


def run(state):
    s, c = state, state.case
    if c["kind"] == "attention":
        if not own:
            return _plain_attention(s)
        s.layer.forward(s.q, s.k, s.v, s.log_decay, s.o, state=s.state, state_out=s.state_out, lengths=s.lengths)
        out = {"o": s.o, "state": s.state_out}
        if c["op"] == "train":
            s.layer.backward(s.q, s.k, s.v, s.log_decay, s.do, s.dq, s.dk, s.dv, state=s.state, dstate_out=s.dstate_out, dstate=s.dstate, lengths=s.lengths)
            out.update(dq=s.dq, dk=s.dk, dv=s.dv, dstate=s.dstate)
        return out
    if c["kind"] == "dropout":
        if not own:
            return {n: _plain_dropped(x, c["p"], s.seed, s.offset).to(x.dtype) for n, x in (("y", s.x), ("dx", s.dy))}
        from paper_1503_02852_amd import layers
        layers.dropout(s.x, s.y, c["p"], s.seed, s.offset)
        layers.dropout(s.dy, s.dx, c["p"], s.seed, s.offset)
        return {"y": s.y, "dx": s.dx}
    if not own:
        return _plain_norm(s)
    if c["op"] == "backward":
        s.layer.backward(s.dy, s.h, s.rstd, gain=s.gain, dh=s.dh, dx=s.dx, dresidual=s.dresidual, dgain=s.dgain)
        out = {"dx": s.dx, "dgain": s.dgain}
        if s.dresidual is not None:
            out["dresidual"] = s.dresidual
        return out
    if c["op"] == "e4m3":
        s.layer.forward_e4m3(s.x, s.y, s.scales, residual=s.residual, gain=s.gain, h=s.h, group=c["group"])
        return {"h": s.h, "y": s.y, "scales": s.scales}
    s.layer.forward(s.x, s.y, residual=s.residual, gain=s.gain, h=s.h, rstd=s.rstd)
    return {"h": s.h, "y": s.y, "rstd": s.rstd}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------
def _exact_attention(s):
    """Frame by frame: S <- decay S + k v^T, o = scale S^T q; the gradient of S back through the frames."""
    c = s.case
    T, N, H, rep = c["T"], c["N"], c["heads"], c["heads"] // c["kv_heads"]
    q, k, v = s.q.double(), s.k.double().repeat_interleave(rep, 2), s.v.double().repeat_interleave(rep, 2)
    decay = torch.exp(s.log_decay.double())[None, :, None, None]
    zeros = torch.zeros(N, H, c["dk"], c["dv"], dtype=torch.float64, device=DEV)
    S = zeros.clone() if s.state is None else s.state.double()
    L = torch.from_numpy(s.lengths_host).to(DEV)
    o = torch.zeros(T, N, H, c["dv"], dtype=torch.float64, device=DEV)
    train = c["op"] == "train"
    if train:
        do = s.do.double()
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for t in range(T):
        there = (t < L)[:, None, None]
        new = S * decay + k[t][..., None] * v[t][..., None, :]
        S = torch.where(there[..., None], new, S) if c["ragged"] else new
        o[t] = torch.where(there, s.scale * torch.matmul(q[t][..., None, :], S)[..., 0, :], o[t])
        if train:
            dq[t] = torch.where(there, s.scale * torch.matmul(S, do[t][..., None])[..., 0], dq[t])
    out = {"o": o, "state": S}
    if not train:
        return out
    G = zeros if s.dstate_out is None else s.dstate_out.double()
    for t in range(T - 1, -1, -1):
        there = (t < L)[:, None, None]
        here = G + s.scale * q[t][..., None] * do[t][..., None, :]
        dk[t] = torch.where(there, torch.matmul(here, v[t][..., None])[..., 0], dk[t])
        dv[t] = torch.where(there, torch.matmul(k[t][..., None, :], here)[..., 0, :], dv[t])
        G = torch.where(there[..., None], here * decay, G)
    shared = lambda x: x.view(T, N, c["kv_heads"], rep, x.shape[-1]).sum(3)  # noqa: E731
    out.update(dq=dq, dk=shared(dk), dv=shared(dv), dstate=G)
    return out


def _exact_factor(rows, dim, p, seed, offset):
    """0 or 1 / (1 - p) for every element, from the generator's definition, with numpy's unsigned words."""
    cut = _threshold(p)
    if cut == 0:
        return torch.ones(rows, dim, dtype=torch.float64, device=DEV)
    groups = (dim + 7) // 8
    index = np.arange(rows * groups, dtype=np.uint64)
    word = np.uint64(0xFFFFFFFF)
    shift = np.uint64(32)
    a, b = index & word, index >> shift
    x, y = np.uint64(offset) & word, np.uint64(offset) >> shift
    x, y = np.full_like(a, x), np.full_like(a, y)
    k0, k1 = seed % 2 ** 32, seed // 2 ** 32
    for _ in range(7):
        left, right = a * np.uint64(0xD2511F53), x * np.uint64(0xCD9E8D57)
        a, b, x, y = (right >> shift) ^ b ^ np.uint64(k0), right & word, (left >> shift) ^ y ^ np.uint64(k1), left & word
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    numbers = np.empty((rows * groups, 8), np.int32)
    for n, w in enumerate((a, b, x, y)):
        numbers[:, 2 * n], numbers[:, 2 * n + 1] = w & np.uint64(0xFFFF), w >> np.uint64(16)
    kept = torch.from_numpy(numbers.reshape(rows, groups * 8)[:, :dim] >= cut).to(DEV)
    return kept.double() * (65536.0 / (65536 - cut))


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "attention":
        return _exact_attention(s)
    factor = _exact_factor(c["rows"], c["dim"], c["p"], s.seed, s.offset)
    if c["kind"] == "dropout":
        return {"y": s.x.double() * factor, "dx": s.dy.double() * factor}
    gain = s.gain.double()
    if c["op"] == "backward":
        h, r, dy = s.h.double(), s.rstd.double()[:, None], s.dy.double()
        dh = s.dh.double() + r * gain * dy - r ** 3 * h * (gain * dy * h).sum(1, keepdim=True) / c["dim"]
        out = {"dx": dh * factor, "dgain": (dy * h * r).sum(0)}
        if s.dresidual is not None:
            out["dresidual"] = dh
        return out
    h = s.x.double() * factor + (0 if s.residual is None else s.residual.double())
    r = 1 / ((h * h).sum(1) / c["dim"] + EPS).sqrt()
    y = h * r[:, None] * gain
    if c["op"] == "forward":
        return {"h": h, "y": y, "rstd": r}
    width = 128 if c["group"] else c["dim"]
    scales = torch.stack([b.abs().amax(1) for b in y.split(width, 1)], 1) / 448
    scales = torch.where(scales == 0, torch.ones_like(scales), scales)
    return {"h": h, "y": y / scales.repeat_interleave(width, 1)[:, :c["dim"]], "scales": scales}
