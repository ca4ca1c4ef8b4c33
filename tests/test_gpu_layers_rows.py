"""Row layers on the GPU: the widest rows."""
import pytest

from oracle import layers_oracle as lo
from tests.test_gpu_layers import DEV

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dim", [(1 << 31) - 8, (1 << 31) - 4, (1 << 31) - 1])
def test_dropout_of_the_widest_rows(dim):
    from paper_1503_02852_amd import layers
    print(f"[dropout] 1 x {dim}", flush=True)
    x, y = torch.ones(1, dim, device=DEV, dtype=torch.bfloat16), torch.full((1, dim), -7.0, device=DEV, dtype=torch.bfloat16)
    layers.dropout(x, y, 0.5, 9, 3)
    groups = -(-dim // 8)
    for first in (0, groups // 2, groups - 100):
        want = torch.from_numpy(lo.dropout_factor(100, 8, 0.5, 9, 3, first_row=first)).reshape(-1)      # (rows of eight units: a counter's number is the row's)
        got = y[0, 8 * first:8 * first + 800].cpu().double()
        assert torch.equal(got, want[:got.numel()]), first
    assert int((y < 0).sum()) == 0
    half = float((y != 0).sum()) / dim
    assert abs(half - 0.5) < 1e-4      # nine times the deviation of 2^31 draws, 1.1e-5
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [100, 1500, 4096, 9001])
def test_every_output_in_the_place_of_every_input(dim, dtype):
    from paper_1503_02852_amd import layers
    g = torch.Generator(device=DEV).manual_seed(dim)
    rows = 300
    make = lambda: torch.randn(rows, dim, device=DEV, generator=g).to(dtype)  # noqa: E731
    x, res, dy, dh = (make() for _ in range(4))
    h, y, rstd, dx, dr = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty_like(x), torch.empty_like(x)
    layer = layers.AddNorm(rows, dim, dtype=dtype, dropout=0.25, seed=1, device=DEV)
    layer.forward(x, y, residual=res, h=h, rstd=rstd)
    layer.backward(dy, h, rstd, dh=dh, dx=dx, dresidual=dr)
    for first in (0, 1):
        a, b = x.clone(), res.clone()
        out = (a, b) if first else (b, a)
        layer.forward(a, out[0], residual=b, h=out[1])
        assert torch.equal(out[0], y) and torch.equal(out[1], h)
    for i in range(3):
        for j in range(3):
            if i == j:
                continue
            t = [dy.clone(), dh.clone(), h.clone()]
            layer.backward(t[0], t[2], rstd, dh=t[1], dx=t[i], dresidual=t[j])
            assert torch.equal(t[i], dx) and torch.equal(t[j], dr), (i, j)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("dim", [1, 100, 129, 600, 1024, 2048, 4096, 5000, 16384])
def test_e4m3_with_everything(dim, group, dtype):
    """Every type, with gain, dropout, the sum and rstd stored, rows further apart than they are long; the same y as the call that stores it in the inputs' type."""
    import numpy as np
    from paper_1503_02852_amd import layers
    from tests.test_gpu_layers import U, half_step, host, rows_of, sum_bound
    r, rows, seed, p = np.random.default_rng(dim), 5, 77 + dim, 0.25
    x, res, gain = rows_of(r, rows, dim, dtype, dim + 5), rows_of(r, rows, dim, dtype, dim + 8, scale=2.0), torch.from_numpy(r.uniform(0.5, 2.0, dim).astype(np.float32)).to(DEV)
    blocks = -(-dim // 128) if group else 1
    y = torch.full((rows, dim + 9), 0.5, device=DEV).to(torch.float8_e4m3fn)
    h, rstd, scales = torch.full((rows, dim + 3), -7.0, device=DEV, dtype=dtype), torch.empty(rows, device=DEV), torch.empty(rows, blocks, device=DEV)
    layer = layers.AddNorm(rows, dim, dtype=dtype, eps=1e-5, dropout=p, seed=seed, offset=5, device=DEV)
    layer.forward_e4m3(x, y[:, :dim], scales, residual=res, gain=gain, h=h[:, :dim], rstd=rstd, group=group)
    assert (y.float()[:, dim:] == 0.5).all() and (h[:, dim:] == -7.0).all()
    factor = lo.dropout_factor(rows, dim, p, seed, 5)
    H, Y, R = lo.add_norm(host(x), host(res), host(gain), np.float32(1e-5), factor)
    dh = sum_bound(dim, factor, host(x), host(res))
    assert (np.abs(host(h[:, :dim]) - H) <= dh + half_step(dtype) * np.abs(H) + torch.finfo(dtype).tiny).all()
    dr = (U * (dim / 2 + 16) * np.ones(rows) + (dh * np.abs(H)).sum(1) / (H * H).sum(1)) * R      # as in the test of the norm itself
    assert (np.abs(host(rstd) - R) <= dr).all()
    dy = (np.abs(H) * dr[:, None] + dh * R[:, None] + 4 * U * np.abs(H) * R[:, None]) * np.abs(host(gain))
    width = 128 if group else dim
    cut = [slice(b * width, min((b + 1) * width, dim)) for b in range(blocks)]
    most = np.stack([np.abs(Y[:, c]).max(1) for c in cut], 1)
    assert (np.abs(host(scales) - most / 448) <= np.stack([dy[:, c].max(1) for c in cut], 1) / 448 + 2 * U * most / 448).all()
    s = np.repeat(host(scales), width, 1)[:, :dim]
    q = host(y[:, :dim].float())
    # e4m3: half a step of 2^-4 relative, below 2^-6 steps of 2^-9; the quotient's two roundings and the scale's
    assert (np.abs(q * s - Y) <= np.maximum(2.0 ** -4 * np.abs(Y), 2.0 ** -10 * s) * (1 + 2.0 ** -10) + dy + 4 * U * np.abs(Y)).all()
    assert (np.abs(q).max(1) == 448).all()
    want = torch.empty(rows, dim, device=DEV, dtype=dtype)
    h2, rstd2 = torch.empty(rows, dim, device=DEV, dtype=dtype), torch.empty_like(rstd)
    layer.forward(x, want, residual=res, gain=gain, h=h2, rstd=rstd2)
    assert torch.equal(h[:, :dim], h2) and torch.equal(rstd, rstd2)
