"""Calls of the operators on block-scaled formats as programs lay out their buffers: outputs side by side, codes and scales in one buffer."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import mx_reference as ref  # noqa: E402
from test_gpu_mx import Layer, _bf16, _check_norm, _f64, _tools  # noqa: E402


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [1, 73, 300])
def test_packed_projections(T, x8):
    """q, k and v into the columns of one buffer, which also holds 16 columns of something else: the exact results, and the rest as it was."""
    c, rt, mx = _tools()
    Ns = (96, 40, 200)
    layer = Layer(T, 1056, Ns, (8, 16), x8, whole=True)
    packed = torch.full((T, sum(Ns) + 16), 3.0, dtype=torch.bfloat16, device=c.device)
    at = np.concatenate([[8], 8 + np.cumsum(Ns)])
    Ys = [packed[:, i:i + n] for i, n in zip(at, Ns)]
    ws = [mx.workspace(T, 1056, n, 16, c.device, x8) for n in Ns]
    descs = [mx.linear_desc(layer.plan, layer.Xt, W, Y, t, w, layer.Xq) for (W, t), Y, w in zip(layer.proj, Ys, ws)]
    mx.lora_mx_linear_multi(c.handle, layer.plan.struct, descs, rt._stream())
    for Y, (want, _, _) in zip(Ys, layer.ref):
        assert torch.equal(Y.cpu(), _bf16(want)[1])
    assert (packed[:, :8] == 3).all() and (packed[:, at[-1]:] == 3).all()


def test_norm_outputs_and_held_rows_side_by_side():
    """H and Y as halves of one buffer; the 8-bit rows and their scales as rows of another."""
    c, rt, mx = _tools()
    for rows, K in ((1, 4096), (37, 1024), (300, 96)):
        x, r, g = (torch.randn(s, device=c.device).bfloat16() for s in ((rows, K), (rows, K), (K,)))
        both = torch.full((rows, 2 * K + 16), 3.0, dtype=torch.bfloat16, device=c.device)
        h, y = both[:, :K], both[:, K:2 * K]
        held = torch.full((rows, K + K // 32 // 16 * 16 + 32), 77, dtype=torch.uint8, device=c.device)
        q = mx.MxTensor(held[:, :K], held[:, K:K + K // 32], "e4m3")
        assert q.codes.data_ptr() == held.data_ptr() and q.scales.data_ptr() == held.data_ptr() + K
        mx.lora_rms_norm(c.handle, mx.norm_desc(x, g, 1e-5, residual=r, h=h, y=y, q=q), rt._stream())
        apart = mx.rms_norm(c, x, g, 1e-5, r, quantize=True)
        assert torch.equal(h, apart.h) and torch.equal(y, apart.y) and torch.equal(q.codes, apart.q.codes) and torch.equal(q.scales, apart.q.scales)
        assert (both[:, 2 * K:] == 3).all() and (held[:, K + K // 32:] == 77).all()
        _check_norm(h, y, _f64(x), _f64(r), _f64(g), 1e-5, "bf16")
        for fmt, width in (("e4m3", K), ("e2m1", K // 2)):
            held.fill_(77)
            q = mx.MxTensor(held[:, :width], held[:, width:width + K // 32], fmt)
            mx.quantize(c, x, fmt, out=q)
            codes, scales = ref.quantize(_f64(x), fmt)
            assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), scales)
            assert (held[:, width + K // 32:] == 77).all()
            assert np.array_equal(_f64(mx.dequantize(c, q)), ref.dequantize(codes, scales, fmt))


def test_no_rows():
    c, rt, mx = _tools()
    x, g = torch.empty(0, 64, dtype=torch.bfloat16, device=c.device), torch.ones(64, dtype=torch.bfloat16, device=c.device)
    pl = rt.plan(c, np.zeros(1, np.int32), np.zeros(1, np.int32), np.array([8], np.int32))
    W = mx.quantize(c, torch.randn(40, 64, device=c.device), "e2m1")
    for q8 in (False, True):
        n = mx.rms_norm(c, x, g, 1e-5, x, quantize=q8)
        assert n.y.shape == n.h.shape == (0, 64) and (n.q is None) == (not q8)
        assert mx.rms_norm(c, x, g, 1e-5, quantize=True, normed=False).q.shape == (0, 64)
        h, outs = mx.norm_linear_multi(c, pl, x, x, g, 1e-5, [(W, None), (W, None)], x8=q8)
        assert h.shape == (0, 64) and all(Y.shape == (0, 40) for Y in outs)
    assert mx.dequantize(c, mx.quantize(c, x, "e2m1")).shape == (0, 64)


@pytest.mark.parametrize("x8", [False, True])
def test_one_workspace_for_every_batch(x8):
    """Sized once for the largest batch, as a serving loop does; what lies behind it stays as it was."""
    c, rt, mx = _tools()
    K, N, most = 2080, 264, 1500
    n = mx.lora_mx_linear_workspace_bytes(most, K, N, 24, int(x8))
    room = torch.full((n + 4096,), 255, dtype=torch.uint8, device=c.device)
    for T in (most, 700, 391, 300, 129, 128, 100, 17, 1):
        layer = Layer(T, K, [N], (8, 24), x8, whole=True)
        for expand in (-1, 0, 1):
            c.set_option("expand_split", expand)
            try:
                Y = mx.linear(c, layer.plan, layer.Xt, *layer.proj[0], Xq=layer.Xq, ws=room[:n])
            finally:
                c.set_option("expand_split", -1)
            assert torch.equal(Y.cpu(), _bf16(layer.ref[0][0])[1]), T
        assert (room[n:] == 255).all()


def test_smallest_workspace():
    """The smallest workspace that is taken, found by its refusals: K in one stretch, the exact result, nothing behind it touched."""
    c, rt, mx = _tools()
    for T, K, N in ((391, 4128, 264), (160, 2080, 40), (100, 1056, 40)):
        for x8 in (False, True):
            layer = Layer(T, K, [N], (8, 24), x8, whole=True)
            W, table = layer.proj[0]
            hi = mx.lora_mx_linear_workspace_bytes(T, K, N, 24, int(x8))
            room = torch.full((hi + 4096,), 255, dtype=torch.uint8, device=c.device)
            Y = torch.zeros(T, N, dtype=torch.bfloat16, device=c.device)
            status = lambda n: mx.lora_mx_linear(None, layer.plan.struct, mx.linear_desc(layer.plan, layer.Xt, W, Y, table, room[:n], layer.Xq), 0, raw=True)  # noqa: E731
            lo = 0  # (no context: nothing is launched)
            while lo < hi:
                mid = (lo + hi) // 2
                lo, hi = (mid + 1, hi) if status(mid) == rt.B.LORA_ERR_WORKSPACE_TOO_SMALL else (lo, mid)
            mx.linear(c, layer.plan, layer.Xt, W, table, Xq=layer.Xq, Y=Y, ws=room[:lo])
            assert torch.equal(Y.cpu(), _bf16(layer.ref[0][0])[1]) and (room[lo:] == 255).all()


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [1, 31, 128, 150, 420])
def test_projections_with_and_without_adapters(T, x8):
    """Some of the projections have a table and some have none, the first one either way; the term in the tiles and from memory."""
    c, rt, mx = _tools()
    layer = Layer(T, 1056, (64, 200, 33, 40), (8, 16, 512), x8, whole=True)
    for have in ((0, 2), (1,), (1, 3), (0, 1, 2, 3), ()):
        for expand in (-1, 0, 1):
            c.set_option("expand_split", expand)
            try:
                outs = mx.linear_multi(c, layer.plan, layer.Xt, [(W, t if i in have else None) for i, (W, t) in enumerate(layer.proj)], Xq=layer.Xq)
            finally:
                c.set_option("expand_split", -1)
            for i, (Y, (W, _), (want, S, _)) in enumerate(zip(outs, layer.proj, layer.ref)):
                assert S.max() < 2 ** 24
                if i not in have:
                    want = layer.Xb @ ref.dequantize(W.codes.cpu().numpy(), W.scales.cpu().numpy(), "e2m1").T
                assert torch.equal(Y.cpu(), _bf16(want)[1]), (have, expand, i)


@pytest.mark.parametrize("T", [1, 90, 300])
def test_inputs_beside_the_output(T):
    """A buffer whose rows hold the 8-bit codes, their scales, the bf16 activations and the output, one behind the other: what is read past
    the end of a row's codes is the output that is being written."""
    c, rt, mx = _tools()
    K, N = 544, 72
    layer = Layer(T, K, [N], (8, 16), True, whole=True)
    at = {"Y": K, "scales": K + 2 * N, "X": K + 2 * N + 32}
    width = at["X"] + 2 * K + 32
    buf = torch.full((T, width), 255, dtype=torch.uint8, device=c.device)
    wide = buf.view(torch.bfloat16)
    Y, X = wide[:, at["Y"] // 2:at["Y"] // 2 + N], wide[:, at["X"] // 2:at["X"] // 2 + K]
    X.copy_(layer.Xt)
    buf[:, :K], buf[:, at["scales"]:at["scales"] + K // 32] = layer.Xq.codes, layer.Xq.scales
    Xq = mx.MxTensor(buf[:, :K], buf[:, at["scales"]:at["scales"] + K // 32], "e4m3")
    assert Xq.codes.data_ptr() == buf.data_ptr() and Xq.scales.data_ptr() == buf.data_ptr() + at["scales"]
    before = buf.clone()
    mx.linear(c, layer.plan, X, *layer.proj[0], Xq=Xq, Y=Y)
    assert torch.equal(Y.cpu(), _bf16(layer.ref[0][0])[1])
    buf[:, at["Y"]:at["Y"] + 2 * N] = before[:, at["Y"]:at["Y"] + 2 * N]
    assert torch.equal(buf, before)
