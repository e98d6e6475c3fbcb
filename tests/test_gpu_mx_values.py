"""The layer on a 4-bit backbone with values that the small whole numbers and unit normals of test_gpu_mx.py do not have: activations that need
both 8-bit parts, blocks of a wide range, infinities and NaN in activations and in adapters."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import mx_reference as ref  # noqa: E402
from test_gpu_mx import BF16, Layer, _bf16, _f64, _tools  # noqa: E402


class Bare:
    """A layer without adapters on given activations; `blind`: weights are zero for every block's first value."""

    def __init__(self, X, Ns, seed=0, blind=False):
        c, rt, mx = _tools()
        rng = np.random.default_rng([seed, *X.shape])
        T, K = X.shape
        self.X, x = _bf16(X)
        assert np.array_equal(self.X, X, equal_nan=True)
        self.Xt = x.to(c.device)
        self.plan = rt.plan(c, np.array([-1], np.int32), np.array([T], np.int32), np.array([8], np.int32))
        self.W, self.held = [], []
        for N in Ns:
            codes = rng.integers(0, 256, (N, K // 2)).astype(np.uint8)
            scales = np.full((N, K // 32), 127, np.uint8)
            if blind:
                codes[:, ::16] &= 0xf0
            self.W.append(ref.dequantize(codes, scales, "e2m1"))
            self.held.append(mx.MxTensor(torch.from_numpy(codes).to(c.device), torch.from_numpy(scales).to(c.device), "e2m1"))

    def run(self, ws=None):
        c, rt, mx = _tools()
        if len(self.held) == 1:
            return [mx.linear(c, self.plan, self.Xt, self.held[0], None, ws=ws)]
        return mx.linear_multi(c, self.plan, self.Xt, [(W, None) for W in self.held])


def eight_bits(rng, T, K):
    """Odd whole numbers up to 255 with 8 significant bits, of either sign: 129 .. 255, and in every block one above 224, so that its scale
    is 1 and what the first 8-bit part (steps of 8 and 16 there) leaves is never zero."""
    x = rng.integers(64, 128, (T, K)) * 2 + 1
    x[:, ::32] = rng.integers(112, 128, x[:, ::32].shape) * 2 + 1
    return x * rng.choice([-1.0, 1.0], (T, K))


def test_the_second_part_is_never_zero():
    x = eight_bits(np.random.default_rng(0), 20, 256)
    codes, scales = ref.quantize(x, "e4m3")
    assert (scales == 127).all() and (ref.dequantize(codes, scales, "e4m3") != x).all()


# (exact: products are multiples of 1/2, and the magnitudes that are added up -- both parts' -- stay below 2^23)
def _check_exact(layer, Ys):
    for Y, W in zip(Ys, layer.W):
        assert ((np.abs(layer.X) + 16) @ np.abs(W).T).max() < 2 ** 23
        assert torch.equal(Y.cpu(), _bf16(layer.X @ W.T)[1]), np.argwhere(_f64(Y) != _bf16(layer.X @ W.T)[0])[:5]


@pytest.mark.parametrize("tile", [0, 1, 2, 3])
@pytest.mark.parametrize("T,K,N", [(129, 32, 40), (257, 128, 300), (300, 544, 513), (200, 1600, 260), (700, 2080, 270), (513, 4128, 257), (260, 1536, 256)])
def test_both_parts_in_every_tile_and_split(T, K, N, tile):
    """Superstages that end inside (K no multiple of 512) and whole ones."""
    c, rt, mx = _tools()
    layer = Bare(eight_bits(np.random.default_rng(T), T, K), [N])
    ws = torch.full((mx.lora_mx_linear_workspace_bytes(T, K, N, 128, 0) + 8 * T * (N + 7) * 4 + 4096,), 255, dtype=torch.uint8, device=c.device)
    try:
        c.set_option("mx_tile", tile)
        for splits in (1, 2, 3, 5, 8):
            c.set_option("mx_split_k", splits)
            _check_exact(layer, layer.run(ws))
    finally:
        c.set_option("mx_tile", -1)
        c.set_option("mx_split_k", -1)


@pytest.mark.parametrize("T", [1, 40, 128, 129, 300, 1100])
def test_eight_significant_bits(T):
    """The built-in choices; several projections share one pair of parts."""
    x = eight_bits(np.random.default_rng(T), T, 1056)
    for Ns in ([72], [64, 200, 33]):
        layer = Bare(x, Ns)
        _check_exact(layer, layer.run())


@pytest.mark.parametrize("T", [3, 100, 128, 140, 300])
def test_blocks_of_a_wide_range(T):
    """Every block holds values from its largest down to 2^-40 of it; the weights leave the largest itself out, so that the small ones are
    seen.  Up to 128 rows the activations are bf16 itself; above, what is at least 2^-6 of the block's scale is exact and the rest off by at
    most 2^-14 of it.  Sums as in test_gpu_mx.py."""
    rng = np.random.default_rng(T)
    K = 1056
    x = (1 + rng.integers(0, 128, (T, K)) / 128) * np.exp2(-rng.integers(5, 41, (T, K))) * rng.choice([-1.0, 1.0], (T, K))
    x[:, ::32] = np.where(rng.random((T, K // 32)) < 0.5, 1.7578125, 1.9921875)  # (just above 224 scales, and well above)
    x *= np.exp2(rng.integers(-3, 4, (T, K // 32))).repeat(32, 1)
    layer = Bare(x, [72], blind=True)
    (Y,), W = layer.run(), layer.W[0]
    assert (W[:, ::32] == 0).all()
    s = np.exp2(ref.quantize(x, "e4m3")[1].astype(float) - 127).repeat(32, 1)
    off = np.where(np.abs(x) >= s * 2.0 ** -6, 0.0, s * 2.0 ** -14) if T > 128 else np.zeros_like(x)
    want, S = x @ W.T, np.abs(x) @ np.abs(W).T
    bound = BF16 * np.abs(want) + (off @ np.abs(W).T + (K / 16 + 64) * 2.0 ** -24 * S) * (1 + BF16)
    assert (np.abs(_f64(Y) - want) <= bound).all(), (np.abs(_f64(Y) - want) / bound).max()


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("T", [1, 9, 100, 128, 129, 200, 1100])
def test_not_finite_activations_stay_in_their_rows(T, value):
    """bf16 activations: rows that hold an infinity or a NaN are infinite or NaN in every column whose weight there is not zero, the others exact."""
    K = 1056
    rng = np.random.default_rng(T)
    x = rng.integers(-4, 5, (T, K)).astype(float)
    layer = Bare(x, [72, 40])
    want = [_bf16(x @ W.T)[1] for W in layer.W]
    bad = sorted({0, T // 2, T - 1})
    for t, k in zip(bad, (5, 640, K - 1)):
        layer.Xt[t, k] = value
    rest = [t for t in range(T) if t not in bad]
    for Y, w, W in zip(layer.run(), want, layer.W):
        Y = Y.cpu()
        for t, k in zip(bad, (5, 640, K - 1)):
            used = torch.from_numpy(W[:, k] != 0)
            assert used.any() and not torch.isfinite(Y[t][used]).any()
        assert torch.equal(Y[rest], w[rest])


RANKS = (16, 16, 8, 8, 8, 24, 40, 16)


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T,tile,expand", [(600, 0, 0), (600, 1, 0), (600, 2, 0), (600, 3, 0), (600, -1, 1), (600, -1, -1), (100, -1, 0), (100, -1, 1), (9, -1, -1)])
def test_an_adapter_that_is_not_finite(T, tile, expand, x8):
    """Infinities and NaN in one adapter: its own rows turn infinite or NaN and no other row changes by a bit -- but that, above 128 rows and for B_a, rows
    that share a block of 16 in the plan's order with them may (0 times infinity in the tiles)."""
    from gpu_common import plan_reference
    c, rt, mx = _tools()
    K, N, ranks = 544, 261, np.asarray(RANKS, np.int32)
    rng = np.random.default_rng(5)
    ids = np.r_[np.arange(len(RANKS)), -1, np.arange(len(RANKS))].astype(np.int32)[:T]
    ntok = np.maximum(rng.multinomial(max(T - len(ids), 0), np.full(len(ids), 1 / len(ids))), 1).astype(np.int32)
    ntok[0] += T - ntok.sum()
    layer = Layer(T, K, [N], RANKS, x8, seed=9)
    pl = rt.plan(c, ids, ntok, ranks)
    W, table = layer.proj[0]
    perm = np.asarray(plan_reference(ids, ntok, ranks)["perm"])
    owner = np.repeat(ids, ntok)[perm]  # adapter of every slot

    def changed(A, Bw):
        Y = mx.linear(c, pl, layer.Xt, W, rt.AdapterTable(A, Bw, table.scales.cpu().numpy(), c.device), Xq=layer.Xq)
        return Y, ~(Y.view(torch.int16) == clean).all(dim=1).cpu().numpy()[perm]

    try:
        c.set_option("mx_tile", tile)
        c.set_option("expand_split", expand)
        if tile >= 0:
            c.set_option("mx_split_k", 1)
        clean = mx.linear(c, pl, layer.Xt, W, table, Xq=layer.Xq).view(torch.int16)
        for bad in range(len(RANKS)):
            mine = owner == bad
            near = np.isin(np.arange(T) // 16, np.unique(np.flatnonzero(mine) // 16)) if T > 128 else mine
            rows = torch.from_numpy(perm[mine]).to(c.device)
            for where in "AB":
                lists = {"A": list(table.A), "B": list(table.B)}
                t = lists[where][bad] = lists[where][bad].clone()
                t[::3] = float("inf")
                t[1::3] = float("nan")
                Y, other = changed(lists["A"], lists["B"])
                assert not (other & ~(near if where == "B" else mine)).any(), (bad, where, owner[other])
                own = Y[rows]
                if where == "B":
                    own = torch.cat([own[:, ::3], own[:, 1::3]], 1)
                assert not torch.isfinite(own).any(), (bad, where)
    finally:
        for name in ("mx_tile", "expand_split", "mx_split_k"):
            c.set_option(name, -1)
