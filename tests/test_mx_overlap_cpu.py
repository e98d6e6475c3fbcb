"""include/lora_mx.h: what counts as an overlap.  Rows of one stride side by side in a buffer do not overlap; a byte in common does.
No GPU: every call is refused, or would be for its missing context alone, before anything is dereferenced."""
import pytest

from paper_2505_14468_amd import binding as B
from paper_2505_14468_amd import mx

AT = [(i + 1) << 44 for i in range(12)]
T, K, NS = 200, 64, (40, 8, 72)
LD = sum(NS)  # of a buffer that holds the outputs side by side


def rows(at, ld, scales, lds, fmt=mx.LORA_MX_E4M3):
    return mx.lora_mx_rows_t(at, ld, scales, lds, fmt, 0)


def plan():
    p = B.lora_plan_t()
    p.T, p.n_req, p.n_adapters, p.r_max, p.magic, p.unit_rows, p.scalars = T, 1, 0, 0, 0x4c6f5241, 16, AT[9]
    return p


def linear(i, Y, ldy=LD, **kw):
    f = dict(K=K, N=NS[i], flags=0, reserved=0, X=AT[0], ldx=K, Xq=rows(AT[1], K, AT[2], 4), W=rows(AT[3] + (i << 36), 32, AT[4] + (i << 36), 4, mx.LORA_MX_E2M1),
             Y=Y, ldy=ldy, tbl=None, ws=AT[6] + (i << 36), wsb=1 << 30)
    f.update(kw)
    return mx.lora_mx_linear_desc(*f.values())


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    import fake_hip
    return fake_hip.build(tmp_path_factory.mktemp("fake_hip"))


def test_outputs_side_by_side_are_launched(fake):
    """Packed projections, below and above 128 rows; H and Y of a norm as halves of one buffer; codes with their scales behind them."""
    import fake_hip
    fake_hip.run(fake, """
        from paper_2505_14468_amd import mx
        K, ns = 64, (40, 8, 72)
        rows = lambda at, ld, scales, lds, fmt: mx.lora_mx_rows_t(at, ld, scales, lds, fmt, 0)
        for T in (73, 300):
            plan = make_plan([-1], [T], [8])
            Y, ld = mem(T * sum(ns) * 2), sum(ns)
            X = mem(T * K * 2)
            descs = []
            for i, n in enumerate(ns):
                size = mx.lora_mx_linear_workspace_bytes(T, K, n, 8, 0)
                descs.append(mx.lora_mx_linear_desc(K, n, 0, 0, X, K, mx.lora_mx_rows_t(), rows(mem(n * K), K // 2, mem(n * 4), 4, 0), Y + 2 * sum(ns[:i]), ld, None, mem(size), size))
            F.fake_reset()
            assert mx.lora_mx_linear_multi(ctx, plan, descs, 0, raw=True) == 0 and F.fake_launches() > 0
            # X beside Y in one buffer
            both = mem(T * (K + 40) * 2)
            d = descs[0]
            d.X, d.ldx, d.Y, d.ldy = both, K + 40, both + 2 * K, K + 40
            assert mx.lora_mx_linear(ctx, plan, d, 0, raw=True) == 0
        n, Kn = 9, 256
        buf = mem(n * 2 * Kn * 2 + n * (Kn + 16))
        held = buf + n * 2 * Kn * 2
        q = rows(held, Kn + 16, held + Kn, Kn + 16, 1)
        norm = mx.lora_rms_norm_desc(1, Kn, n, 1e-5, 0, mem(n * Kn * 2), Kn, mem(n * Kn * 2), Kn, mem(Kn * 2), buf, 2 * Kn, buf + 2 * Kn, 2 * Kn, q)
        assert mx.lora_rms_norm(ctx, norm, 0, raw=True) == 0
        c = mx.lora_mx_convert_desc(1, Kn, n, buf, 2 * Kn, q)
        assert mx.lora_mx_quantize(ctx, c, 0, raw=True) == 0 and mx.lora_mx_dequantize(ctx, c, 0, raw=True) == 0
    """)


def test_a_byte_in_common_is_refused(fake):
    """Two outputs of one stride anywhere near each other: refused if and only if they have a byte in common, in either order; of
    other strides, if their extents meet."""
    import fake_hip
    fake_hip.run(fake, """
        from paper_2505_14468_amd import mx
        T, K, N0, N1, ld = 9, 64, 40, 16, 96
        rows = lambda at, ld, scales, lds, fmt: mx.lora_mx_rows_t(at, ld, scales, lds, fmt, 0)
        plan = make_plan([-1], [T], [8])
        X, W, S = mem(T * K * 2), mem(40 * K), mem(40 * 4)
        size = mx.lora_mx_linear_workspace_bytes(T, K, 40, 8, 0)
        ws = [mem(size), mem(size)]
        span = T * ld * 2
        Y = mem(6 * span) + 2 * span
        def call(at, ld1):
            d = [mx.lora_mx_linear_desc(K, n, 0, 0, X, K, mx.lora_mx_rows_t(), rows(W, K // 2, S, 4, 0), y, l, None, w, size)
                 for y, l, n, w in ((Y, ld, N0, ws[0]), (at, ld1, N1, ws[1]))]
            F.fake_reset()
            a, b = (mx.lora_mx_linear_multi(ctx, plan, e, 0, raw=True) for e in (d, d[::-1]))
            assert a == b and (F.fake_launches() > 0) == (a == 0)
            return a
        first = np.zeros(6 * span, bool)
        for t in range(T):
            first[2 * span + t * ld * 2:][:N0 * 2] = True
        seen = set()
        for ld1 in (ld, ld + 8):
            for off in range(-span - 64, span + 64, 16):
                own = np.zeros(6 * span, bool)
                for t in range(T):
                    own[2 * span + off + t * ld1 * 2:][:N1 * 2] = True
                shared = bool((first & own).any())
                if ld1 != ld:
                    a, b = np.flatnonzero(first), np.flatnonzero(own)
                    shared = a[0] <= b[-1] and b[0] <= a[-1]
                assert call(Y + off, ld1) == (-1 if shared else 0), (ld1, off)
                seen.add(shared)
        assert seen == {False, True}
        n, Kn = 9, 256
        h = mem(8 * n * Kn * 2) + 4 * n * Kn
        def norm(y, ld=2 * Kn):
            d = mx.lora_rms_norm_desc(1, Kn, n, 1e-5, 0, X, Kn, None, 0, W, h, 2 * Kn, y, ld, mx.lora_mx_rows_t())
            return mx.lora_rms_norm(ctx, d, 0, raw=True)
        X, W = mem(n * Kn * 2), mem(Kn * 2)
        for k in range(-5, 6):  # (rows of 2 Kn: half a row further is beside, anything between is not)
            assert norm(h + 2 * Kn * k) == (0 if k % 2 else -1) and norm(h + 2 * Kn * k + 16) == norm(h + 2 * Kn * k - 16) == -1
        assert norm(h + 2 * Kn * 2 * n) == 0
    """)


def test_shared_rows_are_refused_as_before():
    call = lambda *d: mx.lora_mx_linear_multi(None, plan(), list(d), None, raw=True)  # noqa: E731
    for d in ([linear(0, AT[5]), linear(1, AT[5])], [linear(0, AT[5]), linear(2, AT[5] + 2 * 32)], [linear(0, AT[5]), linear(1, AT[5] + 2 * 40, ldy=96)],
              [linear(0, AT[5], X=AT[5] + 16)], [linear(0, AT[6] + 512)]):
        assert call(*d) == B.LORA_ERR_INVALID_ARG
