"""The operators on block-scaled formats against their definitions in 64 bits, on the GPU."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import mx_reference as ref  # noqa: E402

BF16 = 2.0 ** -8  # a rounding to bf16, relative


def _tools():
    from gpu_common import ctx, rt
    from paper_2505_14468_amd import mx
    return ctx(), rt, mx


def _f64(t):
    return t.detach().double().cpu().numpy()


def _bf16(a):
    """An array rounded to bf16, and the tensor that holds it."""
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).bfloat16()
    return t.double().numpy(), t


def _values(rng, rows, K, kind):
    x = rng.standard_normal((rows, K))
    if kind == "wide":
        x *= np.exp2(rng.integers(-100, 100, (rows, K // 32)).repeat(32, 1))
    if kind == "ties":  # halves of the formats' steps, and the limits of the scales
        x = rng.integers(-32, 33, (rows, K)) / 8.0 * np.exp2(rng.integers(-3, 4, (rows, K // 32)).repeat(32, 1))
    if kind == "edge":
        x[:, :32] = 0.0
        if K > 32:
            x[0, 33] = np.inf
        if K > 64:
            x[-1, 65] = np.nan
        if K > 96:
            x[:, 96:128] = 1e-39  # (below fp32's normal numbers)
        if K > 128:
            x[:, 128:160] = 3e38
        if K > 160:
            x[:, 160:192] = 0.0
            x[:, 161] = 2.0 ** -120
            x[:, 165] = -0.0
    return x


@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,kind", [(1, 32, "edge"), (3, 96, "edge"), (5, 192, "edge"), (7, 2048, "plain"), (2, 2080, "ties"), (300, 544, "ties"),
                                         (9, 4128, "wide"), (1, 40000 // 32 * 32, "plain"), (4100, 32, "wide")])
def test_conversions_are_exact(rows, K, kind, dtype, fmt):
    c, rt, mx = _tools()
    rng = np.random.default_rng(rows * 7 + K)
    x = torch.from_numpy(_values(rng, rows, K, kind).astype(np.float32))
    x = (x.bfloat16() if dtype == "bf16" else x)
    want_codes, want_scales = ref.quantize(x.double().numpy(), fmt)
    q = mx.quantize(c, x.to(c.device), fmt)
    scales = q.scales.cpu().numpy()
    assert np.array_equal(scales, want_scales)
    good = np.repeat(want_scales != 255, 32, 1)  # (the codes of a NaN block say nothing)
    got, want = ref.unpack(q.codes.cpu().numpy(), fmt), ref.unpack(want_codes, fmt)
    assert np.array_equal(got[good], want[good])
    for out in (torch.bfloat16, torch.float32):
        back = _f64(mx.dequantize(c, q, out))
        # (rounded as fp32 rounds: 3e38 is held as 4 * 2^126 in 4 bits, which fp32 and bf16 round to infinity)
        with np.errstate(over="ignore"):
            value = ref.dequantize(q.codes.cpu().numpy(), scales, fmt).astype(np.float32).astype(np.float64)
        small = np.abs(value) < 2.0 ** -126
        assert np.array_equal(np.isnan(back), np.isnan(value))
        assert np.array_equal(back[~small & good], value[~small & good])
        assert (np.abs(back[small] - value[small]) <= 2.0 ** -126).all()


def test_every_code_and_scale_opens():
    c, rt, mx = _tools()
    for fmt in ("e2m1", "e4m3"):
        n = 16 if fmt == "e2m1" else 256
        one = np.tile((np.arange(256) % n).astype(np.uint8), (255, 1))
        scales = np.tile(np.arange(255, dtype=np.uint8)[:, None], (1, 8))
        codes = ref.pack(one, fmt)
        q = mx.MxTensor(torch.from_numpy(codes).to(c.device), torch.from_numpy(scales).to(c.device), fmt)
        want = ref.dequantize(codes, scales, fmt)
        normal = (np.abs(want) >= 2.0 ** -126) & (np.abs(want) < 2.0 ** 127) | (want == 0) | np.isnan(want)
        for dtype in (torch.bfloat16, torch.float32):
            got = _f64(mx.dequantize(c, q, dtype))
            assert np.array_equal(got[normal], want[normal], equal_nan=True)


def test_conversions_with_strides_leave_the_rest_alone():
    c, rt, mx = _tools()
    rows, K = 37, 352
    for fmt in ("e2m1", "e4m3"):
        wide = torch.randn(rows, K + 40, device=c.device).bfloat16()
        X = wide[:, 8:8 + K]
        width = K // 2 if fmt == "e2m1" else K
        codes = torch.full((rows, width + 48), 77, dtype=torch.uint8, device=c.device)
        scales = torch.full((rows, 24), 78, dtype=torch.uint8, device=c.device)
        q = mx.MxTensor(codes[:, 16:16 + width], scales[:, 4:4 + K // 32], fmt)
        assert q.codes.data_ptr() == codes.data_ptr() + 16 and q.scales.data_ptr() == scales.data_ptr() + 4
        mx.quantize(c, X, fmt, out=q)
        wc, ws = ref.quantize(X.double().cpu().numpy(), fmt)
        assert np.array_equal(q.codes.cpu().numpy(), wc) and np.array_equal(q.scales.cpu().numpy(), ws)
        assert (codes[:, :16] == 77).all() and (codes[:, 16 + width:] == 77).all()
        assert (scales[:, :4] == 78).all() and (scales[:, 4 + K // 32:] == 78).all()
        out = torch.full((rows, K + 16), 5.0, device=c.device)
        mx.dequantize(c, q, out=out[:, 4:4 + K])
        assert np.array_equal(_f64(out[:, 4:4 + K]), ref.dequantize(wc, ws, fmt))
        assert (out[:, :4] == 5).all() and (out[:, 4 + K:] == 5).all()


# ---- norm ------------------------------------------------------------------------------------------------------------------
# fp32 roundings of y: the sum of x and the residual, the products with the row's scale (two numbers of 24 bits) and with gamma: 3 half
# steps; 48 are allowed, as a sum of squares in fp32 would take with 64 terms in a row per thread and a tree of 10 sums.
NORM32 = 48 * 2.0 ** -24


def _check_norm(h, y, x, r, g, eps, dtype):
    round_to = BF16 if dtype == "bf16" else 2.0 ** -24
    wh, wy = ref.rms_norm(x, g, eps, r)
    if h is not None:
        assert (np.abs(_f64(h) - wh) <= (round_to + 2.0 ** -24) * np.abs(wh)).all()
    if y is not None:
        assert (np.abs(_f64(y) - wy) <= (round_to + NORM32) * np.abs(wy) * (1 + BF16)).all()
    return wy


def _check_held(q, wy):
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    v = ref.dequantize(codes, scales, "e4m3")
    s = np.exp2(scales.astype(float) - 127)
    amax = np.abs(wy).reshape(*scales.shape, 32).max(-1)
    lowest = scales == 0
    assert (amax <= 448 * s * (1 + NORM32)).all() and ((amax > 224 * s * (1 - NORM32)) | lowest).all()
    # half a step of e4m3: 2^-4 of the value, or half of the smallest step 2^-9
    step = np.maximum(2.0 ** -4 * np.abs(wy), 2.0 ** -10 * np.repeat(s, 32, 1))
    assert (np.abs(v - wy) <= step + 2 * NORM32 * np.abs(wy) + 1e-45).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 8), (3, 40), (5, 32), (1, 4096), (2, 2048), (2, 2056), (73, 4096), (391, 5120), (7, 8200), (3, 11008), (2, 16416),
                                    (3, 65536), (1025, 1024), (2600, 96), (777, 4096)])
def test_norm(rows, K, dtype):
    c, rt, mx = _tools()
    torch.manual_seed(rows + K)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, r = (3 * torch.randn(rows, K, device=c.device)).to(t), torch.randn(rows, K, device=c.device).to(t)
    g = (1 + 0.3 * torch.randn(K, device=c.device)).to(t)
    x[0, 0] = 1000.0
    for residual in (None, r):
        for q8 in ((False, True) if K % 32 == 0 else (False,)):
            n = mx.rms_norm(c, x, g, 1e-5, residual, quantize=q8)
            assert (n.h is None) == (residual is None) and (n.q is None) == (not q8)
            wy = _check_norm(n.h, n.y, _f64(x), None if residual is None else _f64(r), _f64(g), 1e-5, dtype)
            if q8:
                _check_held(n.q, wy)
                only = mx.rms_norm(c, x, g, 1e-5, residual, quantize=True, normed=False)
                assert only.y is None and torch.equal(only.q.codes, n.q.codes) and torch.equal(only.q.scales, n.q.scales)


def test_norm_of_a_row_does_not_depend_on_the_others():
    c, rt, mx = _tools()
    for K in (96, 1024, 4096, 11008):
        x, g = torch.randn(600, K, device=c.device).bfloat16(), torch.randn(K, device=c.device).bfloat16()
        every = mx.rms_norm(c, x, g, 1e-5, quantize=True)
        for rows in (1, 77, 599):
            some = mx.rms_norm(c, x[:rows], g, 1e-5, quantize=True)
            assert torch.equal(some.y, every.y[:rows]) and torch.equal(some.q.codes, every.q.codes[:rows]) and torch.equal(some.q.scales, every.q.scales[:rows])


def test_norm_rounds_the_8_bit_rows_once():
    """Ten million elements are enough for some to lie nearer to a border between two 8-bit values than half a step of fp32
    (one in 2^21 does): they fall where the formula in 64 bits has them.  Without a residual, whose sum is fp32's."""
    c, rt, mx = _tools()
    torch.manual_seed(5)
    rows, K = 2600, 4096
    x, g = torch.randn(rows, K, device=c.device).bfloat16(), (1 + 0.3 * torch.randn(K, device=c.device)).bfloat16()
    n = mx.rms_norm(c, x, g, 1e-5, quantize=True)
    _, y = ref.rms_norm(_f64(x), _f64(g), 1e-5)
    for i in range(0, rows, 200):
        codes, scales = ref.quantize(y[i:i + 200], "e4m3")
        assert np.array_equal(n.q.codes[i:i + 200].cpu().numpy(), codes) and np.array_equal(n.q.scales[i:i + 200].cpu().numpy(), scales)
    mantissa, exponent = np.frexp(y)  # (a bf16 value has 8 significant bits)
    assert np.array_equal(_f64(n.y), np.ldexp(np.rint(mantissa * 256) / 256, exponent))


def test_norm_special_rows():
    """Rows of zeros, with and without eps; an infinity or a NaN stays in its row; values too small to square."""
    c, rt, mx = _tools()
    K = 256
    x = torch.randn(6, K, device=c.device)
    x[1] = 0.0
    x[2, 7] = float("inf")
    x[3, 9] = float("nan")
    x[4] = 1e-30
    g = torch.ones(K, device=c.device)
    n = mx.rms_norm(c, x, g, 1e-5, quantize=True)
    y = n.y.cpu()
    assert (y[1] == 0).all() and (n.q.scales[1] == 0).all() and (n.q.codes[1] == 0).all()
    assert torch.isnan(y[2, 7]) and (y[2, :7] == 0).all() and (n.q.scales[2, 0] == 255) and (n.q.scales[2, 1:] == 0).all()
    assert torch.isnan(y[3]).all() and (n.q.scales[3] == 255).all()
    for i in (0, 4, 5):
        _check_norm(None, y[i:i + 1], _f64(x[i:i + 1]), None, np.ones(K), 1e-5, "f32")
    bare = mx.rms_norm(c, x[1:2].contiguous(), g, 0.0)
    assert torch.isnan(bare.y).all()  # 0 / 0


def test_norm_in_place_and_strided():
    c, rt, mx = _tools()
    rows, K = 19, 320
    wide = torch.randn(rows, K + 64, device=c.device).bfloat16()
    x, r = wide[:, 16:16 + K], torch.randn(rows, K, device=c.device).bfloat16()
    g = torch.randn(K, device=c.device).bfloat16()
    X, R = _f64(x), _f64(r)
    before = wide.clone()
    # H over the residual, Y over the input
    mx.lora_rms_norm(c.handle, mx.norm_desc(x, g, 1e-6, residual=r, h=r, y=x), rt._stream())
    torch.cuda.synchronize()
    _check_norm(r, x, X, R, _f64(g), 1e-6, "bf16")
    assert torch.equal(wide[:, :16], before[:, :16]) and torch.equal(wide[:, 16 + K:], before[:, 16 + K:])


# ---- the layer ---------------------------------------------------------------------------------------------------------------

def _batch(rng, T, n_adapters, bare):
    """Request ids and lengths of T rows."""
    ntok = []
    while sum(ntok) < T:
        ntok.append(int(min(rng.integers(0, 2 + T // 3), T - sum(ntok))) if rng.random() < 0.5 else 1)
    ids = rng.integers(-1 if bare else 0, n_adapters, len(ntok)) if n_adapters else np.full(len(ntok), -1)
    return ids.astype(np.int32), np.array(ntok, np.int32)


class Layer:
    """A layer's inputs on the GPU and in 64 bits."""

    def __init__(self, T, K, Ns, ranks=(), x8=False, whole=False, bare=True, seed=0, special=None):
        c, rt, mx = _tools()
        rng = np.random.default_rng([seed, T, K, *Ns])
        self.T, self.x8 = T, x8
        dev = c.device
        self.ids, self.ntok = _batch(rng, T, len(ranks), bare)
        self.rows = np.repeat(self.ids, self.ntok)
        self.X, x = _bf16(rng.integers(-4, 5, (T, K)) if whole else rng.standard_normal((T, K)))
        self.Xt = x.to(dev)
        self.Xq = None
        self.Xb = self.X
        if x8:
            if whole:  # another set of whole numbers, so that what reads which is seen
                codes, scales = ref.quantize(rng.integers(-7, 8, (T, K)) * np.exp2(rng.integers(0, 3, (T, K // 32))).repeat(32, 1), "e4m3")
            else:
                codes, scales = ref.quantize(self.X, "e4m3")
            self.Xb = ref.dequantize(codes, scales, "e4m3")
            self.Xq = mx.MxTensor(torch.from_numpy(codes).to(dev), torch.from_numpy(scales).to(dev), "e4m3")
        self.proj, self.ref = [], []
        scale = (2.0 ** rng.integers(-2, 3, len(ranks)) if whole else 16.0 / np.array(ranks, float)) if len(ranks) else np.zeros(0)
        for N in Ns:
            codes = rng.integers(0, 256, (N, K // 2)).astype(np.uint8)
            scales = (rng.integers(127, 130, (N, K // 32)) if whole else rng.integers(118, 123, (N, K // 32))).astype(np.uint8)
            if special is not None:
                special(codes, scales)
            W = ref.dequantize(codes, scales, "e2m1")
            A, Bw, At, Bt = [], [], [], []
            for r in ranks:
                if whole:
                    a = np.zeros((r, K))
                    for j in range(r):
                        a[j, rng.integers(0, K, 6)] = rng.choice([-1, 1], 6)
                    b = rng.integers(-2, 3, (N, r))
                else:
                    a, b = rng.standard_normal((r, K)) * K ** -0.5, rng.standard_normal((N, r)) * 0.02
                (a, at), (b, bt) = _bf16(a), _bf16(b)
                A.append(a), Bw.append(b), At.append(at.to(dev)), Bt.append(bt.to(dev))
            table = rt.AdapterTable(At, Bt, scale, dev) if len(ranks) else None
            self.proj.append((mx.MxTensor(torch.from_numpy(codes).to(dev), torch.from_numpy(scales).to(dev), "e2m1"), table))
            self.ref.append(ref.linear(self.Xb, W, self.X, self.rows, A, Bw, scale))
        self.plan = rt.plan(c, self.ids, self.ntok, np.array(ranks, np.int32))

    def run(self):
        c, rt, mx = _tools()
        if len(self.proj) == 1:
            return [mx.linear(c, self.plan, self.Xt, *self.proj[0], Xq=self.Xq)]
        return mx.linear_multi(c, self.plan, self.Xt, self.proj, Xq=self.Xq)


def _check_whole(layer):
    """Whole numbers whose sums stay below 2^24: every partial sum is exact, and Y is the exact result rounded once."""
    for Y, (want, S, _) in zip(layer.run(), layer.ref):
        assert S.max() < 2 ** 24
        _, t = _bf16(want)
        assert torch.equal(Y.cpu(), t), (np.abs(_f64(Y) - want).max(), np.argwhere(_f64(Y) != t.double().numpy())[:5])


def _check_close(layer):
    """bf16 rounding of Y; fp32 sums, at most K / 16 + 64 of them in a row; V rounded to bf16 (batches of many rows or much adapter
    work).  Errors of sums are relative to the magnitudes that are added."""
    K = layer.X.shape[1]
    for Y, (want, S, term) in zip(layer.run(), layer.ref):
        bound = BF16 * np.abs(want) + (K / 16 + 64) * 2.0 ** -24 * S * (1 + BF16) + BF16 * term * (1 + BF16)
        assert (np.abs(_f64(Y) - want) <= bound).all(), (np.abs(_f64(Y) - want) / bound).max()


ROWS = [1, 2, 16, 17, 33, 64, 65, 100, 127, 128, 129, 200, 257, 300]


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", ROWS)
@pytest.mark.parametrize("K,N", [(32, 1), (96, 17), (544, 250), (1056, 40), (2080, 129)])
def test_layer_whole_numbers(T, K, N, x8):
    _check_whole(Layer(T, K, [N], (8, 24), x8, whole=True))


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [1, 20, 70, 128, 140, 500])
def test_layer_without_adapters(T, x8):
    layer = Layer(T, 1184, [72], (), x8, whole=True)
    _check_whole(layer)
    if x8:  # the base product does not read X
        layer.Xt = None
        _check_whole(layer)


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [1, 31, 64, 90, 128, 150, 420])
def test_layer_several_projections(T, x8):
    _check_whole(Layer(T, 1056, [64, 200, 33], (8, 16, 64), x8, whole=True))


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T,K,N,ranks", [(1, 4096, 1000, (16,)), (64, 4096, 512, (16, 8, 64)), (73, 11008, 300, (64, 8)), (128, 2048, 700, (128,) * 9),
                                         (391, 4096, 1030, (16, 32)), (1216, 1024, 520, (8, 16, 32, 64))])
def test_layer_normal_values(T, K, N, ranks, x8):
    _check_close(Layer(T, K, [N], ranks, x8))


@pytest.mark.parametrize("values", [512, 1024])
@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [1, 16, 17, 33, 64, 65, 96, 112, 128])
def test_every_slice(T, x8, values):
    """Decode-sized batches with each length of the backbone's slices and workgroups of 8 to 12 waves; K that ends inside a slice."""
    c, rt, mx = _tools()
    try:
        c.set_option("mx_slice", values)
        for waves, K, N in ((8, 2080, 130), (9, 4128, 200), (11, 1056, 190), (12, 3168, 410)):
            c.set_option("decode_waves", waves)
            c.set_option("expand_split", waves % 2)
            _check_whole(Layer(T, K, [N], (8, 24, 64), x8, whole=True, seed=waves))
    finally:
        for name in ("mx_slice", "decode_waves", "expand_split"):
            c.set_option(name, -1)


@pytest.mark.parametrize("tile", [0, 1, 2, 3])
@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T,K,N", [(129, 32, 40), (257, 128, 300), (300, 544, 513), (200, 1600, 260), (700, 2080, 270), (513, 4128, 257)])
def test_every_tile_and_split(T, K, N, x8, tile):
    """Each tile, whole and split along K into as many stretches as there are superstages of 512 values, up to 8."""
    c, rt, mx = _tools()
    layer = Layer(T, K, [N], (8, 40, 128), x8, whole=True)
    want = _bf16(layer.ref[0][0])[1]
    assert layer.ref[0][1].max() < 2 ** 24
    ws = torch.empty(mx.lora_mx_linear_workspace_bytes(T, K, N, 128, int(x8)) + 8 * T * (N + 7) * 4 + 4096, dtype=torch.uint8, device=c.device)
    try:
        c.set_option("mx_tile", tile)
        for splits in (1, 2, 3, 5, 8):
            for expand in (-1, 0, 1):  # the adapter term: by the batch's own rule, all in the tile, short segments' from memory
                c.set_option("mx_split_k", splits)
                c.set_option("expand_split", expand)
                Y = mx.linear(c, layer.plan, layer.Xt, *layer.proj[0], Xq=layer.Xq, ws=ws)
                assert torch.equal(Y.cpu(), want), (splits, expand, np.argwhere(_f64(Y) != want.double().numpy())[:4])
    finally:
        for name in ("mx_tile", "mx_split_k", "expand_split"):
            c.set_option(name, -1)


@pytest.mark.parametrize("tile", [0, 1, 2, 3])
def test_many_segments_in_a_tile(tile):
    """A row to a segment, and segments of every length, with the whole adapter term in the tile."""
    c, rt, mx = _tools()
    n = 150
    layer = Layer(400, 544, [140], tuple([8, 16, 24, 72][i % 4] for i in range(n)), True, whole=True)
    try:
        c.set_option("mx_tile", tile)
        for expand in (0, 1):
            c.set_option("expand_split", expand)
            _check_whole(layer)
    finally:
        c.set_option("mx_tile", -1)
        c.set_option("expand_split", -1)


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [3, 80, 128, 170])
def test_nan_scale_stays_in_its_column(T, x8):
    """A block whose scale is 255 makes its own column NaN and no other."""
    def special(codes, scales):
        scales[5, 3] = 255
        scales[40, -1] = 255
    layer = Layer(T, 1056, [70], (8,), x8, whole=True, special=special)
    (Y,), (want, _, _) = layer.run(), layer.ref[0]
    bad = np.isnan(want).any(0)
    assert bad.sum() == 2 and torch.isnan(Y[:, 5]).all() and torch.isnan(Y[:, 40]).all()
    assert torch.equal(Y.cpu()[:, ~torch.from_numpy(bad)], _bf16(want[:, ~bad])[1])


@pytest.mark.parametrize("T", [9, 200])
def test_nan_in_a_row_of_activations_stays_in_it(T):
    c, rt, mx = _tools()
    layer = Layer(T, 544, [70], (), True, whole=True)
    want = layer.ref[0][0].copy()
    layer.Xq.codes[4, 100] = 0x7f
    layer.Xq.scales[7, 2] = 255
    (Y,) = layer.run()
    assert torch.isnan(Y[4]).all() and torch.isnan(Y[7]).all()
    rest = [t for t in range(T) if t not in (4, 7)]
    assert torch.equal(Y.cpu()[rest], _bf16(want[rest])[1])


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [5, 128, 200])
def test_strides_and_the_rest_of_the_output(T, x8):
    c, rt, mx = _tools()
    layer = Layer(T, 544, [70], (8,), x8, whole=True)
    W, table = layer.proj[0]
    wide = torch.full((T, 120), 3.0, dtype=torch.bfloat16, device=c.device)
    Y = wide[:, 16:86]
    codes = torch.zeros((70, 544 // 2 + 32), dtype=torch.uint8, device=c.device)
    scales = torch.full((70, 32), 255, dtype=torch.uint8, device=c.device)  # (what follows the scales is not used)
    codes[:, 16:16 + 272], scales[:, 4:21] = W.codes, W.scales
    W2 = mx.MxTensor(codes[:, 16:16 + 272], scales[:, 4:21], "e2m1")
    X = torch.full((T, 600), float("nan"), dtype=torch.bfloat16, device=c.device)
    X[:, 8:552] = layer.Xt
    Xq = None
    if x8:
        xc = torch.full((T, 592), 0x7f, dtype=torch.uint8, device=c.device)
        xs = torch.full((T, 36), 255, dtype=torch.uint8, device=c.device)
        xc[:, 32:576], xs[:, 8:25] = layer.Xq.codes, layer.Xq.scales
        Xq = mx.MxTensor(xc[:, 32:576], xs[:, 8:25], "e4m3")
    mx.linear(c, layer.plan, X[:, 8:552], W2, table, Xq=Xq, Y=Y)
    assert torch.equal(Y.cpu(), _bf16(layer.ref[0][0])[1])
    assert (wide[:, :16] == 3).all() and (wide[:, 86:] == 3).all()


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [40, 300])
def test_workspace_of_other_calls_leaves_nothing_behind(T, x8):
    """The workspace may hold anything: NaN everywhere, then another shape's."""
    c, rt, mx = _tools()
    a, b = Layer(T, 1056, [100], (8, 16), x8, whole=True), Layer(T - 3, 544, [333], (16,), x8, whole=True, seed=1)
    size = max(mx.lora_mx_linear_workspace_bytes(T, 1056, 100, 16, int(x8)), mx.lora_mx_linear_workspace_bytes(T - 3, 544, 333, 16, int(x8)))
    ws = torch.full((size,), 255, dtype=torch.uint8, device=c.device)
    for layer in (a, b, a):
        Y = mx.linear(c, layer.plan, layer.Xt, *layer.proj[0], Xq=layer.Xq, ws=ws)
        assert torch.equal(Y.cpu(), _bf16(layer.ref[0][0])[1])


def test_adapter_of_an_emptied_slot():
    """The rows of an adapter that was evicted behind the plan are the backbone's product or undefined, the others' are right."""
    c, rt, mx = _tools()
    for T in (40, 300):
        for x8 in (False, True):
            layer = Layer(T, 544, [70], (8, 16), x8, whole=True, bare=False)
            layer.proj[0][1].set_slot(0, None, None)
            (Y,) = layer.run()
            st, _ = layer.plan.status(c)
            assert st == rt.B.LORA_ERR_ADAPTER_NOT_RESIDENT
            rest = layer.rows == 1
            assert torch.equal(Y.cpu()[rest], _bf16(layer.ref[0][0][rest])[1])


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [30, 260])
def test_a_plan_that_was_not_built_stores_nothing(T, x8):
    c, rt, mx = _tools()
    layer = Layer(T, 544, [70], (8,), x8, whole=True)
    bad = torch.full((len(layer.ids),), 9, dtype=torch.int32, device=c.device)  # no such adapter
    pl = rt.plan_device(c, bad, torch.from_numpy(layer.ntok).to(c.device), torch.tensor([8], dtype=torch.int32, device=c.device), 8, T)
    Y = torch.full((T, 72), 7.0, dtype=torch.bfloat16, device=c.device)
    mx.linear(c, pl, layer.Xt, *layer.proj[0], Xq=layer.Xq, Y=Y[:, :70])
    assert pl.status(c)[0] == rt.B.LORA_ERR_BAD_ADAPTER_ID and (Y == 7).all()


def test_the_front_of_a_decoder_layer():
    """Norm, 8-bit rows and the projections that read them, as they are called together: against the definitions chained in 64 bits
    on the 8-bit rows that the norm left."""
    c, rt, mx = _tools()
    for T in (1, 73, 200):
        layer = Layer(T, 1024, [256, 64, 64], (8, 32), False, seed=3)
        x, r = layer.Xt, torch.randn(T, 1024, device=c.device).bfloat16()
        g = (1 + 0.2 * torch.randn(1024, device=c.device)).bfloat16()
        for x8 in (True, False):
            h, outs = mx.norm_linear_multi(c, layer.plan, x, r, g, 1e-5, layer.proj, x8=x8)
            n = mx.rms_norm(c, x, g, 1e-5, r, quantize=True)
            assert torch.equal(h, n.h)
            layer.X, layer.Xb = _f64(n.y), _f64(mx.dequantize(c, n.q, torch.float32)) if x8 else _f64(n.y)
            for Y, (W, table) in zip(outs, layer.proj):
                Wv = ref.dequantize(W.codes.cpu().numpy(), W.scales.cpu().numpy(), "e2m1")
                want, S, term = ref.linear(layer.Xb, Wv, layer.X, layer.rows, [_f64(a) for a in table.A], [_f64(b) for b in table.B], _f64(table.scales))
                bound = BF16 * np.abs(want) + (1024 / 16 + 64) * 2.0 ** -24 * S * (1 + BF16) + BF16 * term * (1 + BF16)
                assert (np.abs(_f64(Y) - want) <= bound).all()


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [24, 128, 300])
def test_replayed_graph_equals_eager_calls(T, x8):
    """Norm and layer captured on a side stream, replayed with new activations and another batch of the same sizes in the same buffers."""
    c, rt, mx = _tools()
    layer = Layer(T, 1056, [96, 40], (8, 16), x8, whole=True, bare=False)
    n_req = len(layer.ids)
    dev = c.device
    plan_buf = torch.empty(rt.B.lora_plan_bytes(n_req, T, 2, 16), dtype=torch.uint8, device=dev)
    ids, ntok = torch.from_numpy(layer.ids).to(dev), torch.from_numpy(layer.ntok).to(dev)
    ranks = torch.tensor([8, 16], dtype=torch.int32, device=dev)
    x, g = torch.randn(T, 1056, device=dev).bfloat16(), torch.ones(1056, device=dev).bfloat16()
    y, q = torch.empty_like(x), mx.empty(T, 1056, "e4m3", dev)
    ws = [mx.workspace(T, 1056, N, 16, dev, x8) for N in (96, 40)]
    Ys = [torch.zeros(T, N, dtype=torch.bfloat16, device=dev) for N in (96, 40)]

    def step(pl):
        s = rt._stream()
        mx.lora_rms_norm(c.handle, mx.norm_desc(x, g, 1e-5, y=y, q=q), s)
        descs = [mx.linear_desc(pl, y, W, Y, t, w, q if x8 else None) for (W, t), Y, w in zip(layer.proj, Ys, ws)]
        mx.lora_mx_linear_multi(c.handle, pl.struct, descs, s)

    side = torch.cuda.Stream()
    pl = rt.plan_device(c, ids, ntok, ranks, 16, T, buf=plan_buf)
    step(pl)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rt.plan_device(c, ids, ntok, ranks, 16, T, buf=plan_buf)
        step(pl)
    for k in range(4):
        x.copy_(torch.randn(T, 1056, device=dev))
        ids.copy_(torch.randint(-1, 2, (n_req,), dtype=torch.int32, device=dev))
        graph.replay()
        torch.cuda.synchronize()
        got = [Y.clone() for Y in Ys]
        (torch.randn(1000, 1000, device=dev) @ torch.randn(1000, 1000, device=dev)).sum()
        for Y in Ys:
            Y.zero_()
        step(rt.plan_device(c, ids, ntok, ranks, 16, T, buf=plan_buf))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, Ys)), k
        assert pl.status(c)[0] == 0


@pytest.mark.parametrize("x8", [False, True])
def test_two_graphs_on_one_workspace(x8):
    """Both replayed in turn, with a bigger eager call on the same workspace in between; the outputs are the exact ones every time."""
    c, rt, mx = _tools()
    layers = [Layer(70, 1056, [100], (8, 16), x8, whole=True), Layer(300, 544, [333], (16,), x8, whole=True, seed=1),
              Layer(600, 1056, [264], (24,), x8, whole=True, seed=2)]
    want = [_bf16(a.ref[0][0])[1] for a in layers]
    size = max(mx.lora_mx_linear_workspace_bytes(a.T, a.X.shape[1], want[i].shape[1], 32, int(x8)) for i, a in enumerate(layers))
    ws = torch.full((size,), 255, dtype=torch.uint8, device=c.device)
    Ys = [torch.zeros(w.shape[0], (w.shape[1] + 7) // 8 * 8, dtype=torch.bfloat16, device=c.device)[:, :w.shape[1]] for w in want]
    descs = [mx.linear_desc(a.plan, a.Xt, a.proj[0][0], Y, a.proj[0][1], ws, a.Xq) for a, Y in zip(layers, Ys)]
    run = lambda i: mx.lora_mx_linear(c.handle, layers[i].plan.struct, descs[i], rt._stream())  # noqa: E731
    side, graphs = torch.cuda.Stream(), []
    for i in (0, 1):
        run(i)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            run(i)
    for k in range(3):
        for Y in Ys:
            Y.zero_()
        graphs[k % 2].replay()
        run(2)
        graphs[1 - k % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(Y.cpu(), w) for Y, w in zip(Ys, want)), k


@pytest.mark.parametrize("x8", [False, True])
def test_calls_on_two_streams_at_once(x8):
    """One context, two streams, a workspace each."""
    c, rt, mx = _tools()
    layers = [Layer(90, 1056, [264], (8, 16), x8, whole=True), Layer(700, 1056, [264], (16, 8), x8, whole=True, seed=1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] += layers[i].run()
    torch.cuda.synchronize()
    for layer, ys in zip(layers, got):
        want = _bf16(layer.ref[0][0])[1]
        assert all(torch.equal(Y.cpu(), want) for Y in ys)
