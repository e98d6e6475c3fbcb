"""The root-mean-square norm over the whole range of its types, and its roundings, in every form that the length of a row chooses.

Without a residual fp32's y is the definition's, rounded once: the squares are summed in 64 bits, the row's scale is kept in 48, so that what
is rounded is off by less than 2^-40.  Narrower outputs are rounded once from more bits than fp32's."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import mx_reference as ref  # noqa: E402
from test_gpu_mx import _f64, _tools  # noqa: E402

LENGTHS = [64, 512, 1024, 2048, 4096, 5120, 8192, 16384, 32768, 65536]
ONCE32 = 2.0 ** -24 + 2.0 ** -40


def _check_once(n, x, g, eps):
    """Every output of a norm without a residual is the definition's value, rounded once."""
    with np.errstate(invalid="ignore"):
        _, y = ref.rms_norm(_f64(x), _f64(g), eps)
    assert np.isfinite(y).all()
    big = np.abs(y) >= 2.0 ** -100
    if x.dtype is torch.float32:
        assert (np.abs(_f64(n.y) - y)[big] <= ONCE32 * np.abs(y)[big]).all(), (np.abs(_f64(n.y) - y)[big] / np.abs(y)[big]).max() * 2 ** 24
    else:
        m, e = np.frexp(y)
        assert np.array_equal(_f64(n.y)[big], np.ldexp(np.rint(m * 256) / 256, e)[big])  # (8 significant bits)
    assert (np.abs(_f64(n.y))[~big] <= 2.0 ** -99).all()
    if n.q is not None:
        codes, scales = ref.quantize(y, "e4m3")
        held = ref.dequantize(n.q.codes.cpu().numpy(), n.q.scales.cpu().numpy(), "e4m3")  # (as values: the formula gives zeros of either sign)
        assert np.array_equal(held, ref.dequantize(codes, scales, "e4m3")) and np.array_equal(n.q.scales.cpu().numpy(), scales)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K", LENGTHS)
def test_every_output_is_rounded_once(K, dtype):
    c, rt, mx = _tools()
    torch.manual_seed(K)
    x, g = (3 * torch.randn(400000 // K + 1, K, device=c.device)).to(dtype), (1 + 0.3 * torch.randn(K, device=c.device)).to(dtype)
    _check_once(mx.rms_norm(c, x, g, 1e-5, quantize=True), x, g, 1e-5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K", LENGTHS)
def test_rows_of_any_size(K, dtype):
    """A row's scale may lie outside of fp32's normal numbers, or of fp32 altogether: with eps 0, rows of 2^-130 (multiples of 2^-149 in fp32,
    of 2^-133 in bf16) to 2^125, and one with a single smallest value among zeros."""
    c, rt, mx = _tools()
    torch.manual_seed(K)
    sizes = torch.tensor([2.0 ** e for e in (-130, -128, -125, -121, -119, -100, 0, 90, 99, 101, 119, 121, 125)], dtype=torch.float64)
    x = (torch.randn(len(sizes) + 1, K, dtype=torch.float64).clamp_(-3.9, 3.9))
    x[:-1] *= sizes[:, None]
    x[-1] = 0.0
    x[-1, 5] = 2.0 ** -133 if dtype is torch.bfloat16 else 2.0 ** -149
    x, g = x.to(dtype).to(c.device), (1 + 0.3 * torch.randn(K, device=c.device)).to(dtype)
    assert torch.isfinite(x).all() and (x != 0).any(1).all()
    _check_once(mx.rms_norm(c, x, g, 0.0, quantize=True), x, g, 0.0)
    n = mx.rms_norm(c, x, g, 0.0, residual=torch.zeros_like(x), quantize=True)  # (the sum is exact)
    _check_once(n, x, g, 0.0)
    assert torch.equal(n.h, x)
