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
