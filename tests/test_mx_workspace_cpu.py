"""The workspace of the layer on a 4-bit backbone: the size for T rows serves every batch of up to T rows, of any ranks up to r_max, with 8-bit
activations or without, as a serving loop that sizes it once needs.  No GPU: a call that the workspace is big enough for is
refused for its missing context alone."""
import numpy as np
import pytest

from paper_2505_14468_amd import binding as B
from paper_2505_14468_amd import mx

AT = [(i + 1) << 44 for i in range(12)]
SHAPES = [(11008, 4096, 64), (4096, 11008, 64), (4096, 4096, 16), (4096, 1000, 512), (1056, 40, 8), (32, 8, 8), (8192, 256, 0)]


def call(T, K, N, r_max, xq, nbytes):
    p = B.lora_plan_t()
    p.T, p.n_req, p.n_adapters, p.r_max, p.magic, p.unit_rows, p.scalars = T, 1, 2, r_max, 0x4c6f5241, 16, AT[9]
    rows = lambda at, ld, scales, lds, fmt: mx.lora_mx_rows_t(at, ld, scales, lds, fmt, 0)  # noqa: E731
    table = B.make_adapter_table(2, AT[7], AT[7] + 64, AT[7] + 128)
    ld = (K // 32 + 3) // 4 * 4
    d = mx.lora_mx_linear_desc(K, N, 0, 0, AT[0], K, rows(AT[1], K, AT[2], ld, 1) if xq else mx.lora_mx_rows_t(), rows(AT[3], K // 2, AT[4], ld, 0), AT[5],
                               (N + 7) // 8 * 8, mx.C.pointer(table), AT[6], nbytes)
    return mx.lora_mx_linear(None, p, d, None, raw=True)


@pytest.mark.parametrize("K,N,r_max", SHAPES)
def test_the_size_for_the_largest_batch_serves_the_smaller_ones(K, N, r_max):
    sizes = [1, 5, 16, 17, 100, 127, 128, 129, 160, 200, 256, 257, 300, 391, 512, 513, 700, 1024, 1025, 1216, 1500, 2000, 2048, 2049, 4200, 7500]
    for most in sizes:
        n = mx.lora_mx_linear_workspace_bytes(most, K, N, r_max, 0)
        for T in [t for t in sizes if t <= most]:
            for xq in (0, 1):
                for r in {r_max, r_max // 2}:
                    assert call(T, K, N, r, xq, n) == B.LORA_ERR_INVALID_ARG, (most, T, xq, r)
        n = mx.lora_mx_linear_workspace_bytes(most, K, N, r_max, 1)
        for T in [t for t in sizes if t <= most]:
            assert call(T, K, N, r_max, 1, n) == B.LORA_ERR_INVALID_ARG, (most, T)


@pytest.mark.parametrize("K,N,r_max", SHAPES)
def test_what_is_needed_grows_with_the_batch(K, N, r_max):
    """The smallest workspace that is taken: never more for fewer rows on either side of 128, nor than the size reported."""
    def least(T, xq):
        lo, hi = 0, mx.lora_mx_linear_workspace_bytes(T, K, N, r_max, xq)
        assert call(T, K, N, r_max, xq, hi) == B.LORA_ERR_INVALID_ARG
        while lo < hi:
            mid = (lo + hi) // 2
            lo, hi = (lo, mid) if call(T, K, N, r_max, xq, mid) == B.LORA_ERR_INVALID_ARG else (mid + 1, hi)
        assert lo == 0 or call(T, K, N, r_max, xq, lo - 1) == B.LORA_ERR_WORKSPACE_TOO_SMALL
        return lo

    for xq in (0, 1):
        for part in ((1, 17, 64, 128), (129, 200, 391, 700, 1024, 1025, 1500, 2048, 5000)):
            got = [least(T, xq) for T in part]
            assert got == sorted(got), (part, got)


def test_sizes_of_no_batch():
    f = mx.lora_mx_linear_workspace_bytes
    assert f(2 ** 31, 64, 64, 8, 0) == f(2 ** 62, 4096, 4096, 64, 1) == 0
    assert f(2 ** 20, 64, 64, 8, 0) > 0


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    import fake_hip
    return fake_hip.build(tmp_path_factory.mktemp("fake_hip"))


def test_fewer_stretches_where_there_is_no_room_for_their_sums(fake):
    """391 rows of 11008 -> 4096 are split along K with the reported size, less or not at all with what remains of it."""
    import fake_hip
    fake_hip.run(fake, """
        from paper_2505_14468_amd import mx
        T, K, N = 391, 11008, 4096
        plan = make_plan([-1], [T], [8])
        rows = lambda n, w, fmt: mx.lora_mx_rows_t(mem(n * w), w, mem(n * 344), 344, fmt, 0)
        d = make_desc(plan, K, N)
        full = mx.lora_mx_linear_workspace_bytes(T, K, N, 8, 1)
        one = T * N * 4
        ws = mem(full)
        m = mx.lora_mx_linear_desc(K, N, 0, 0, d.X, d.ldx, rows(T, K, 1), rows(N, K // 2, 0), d.Y, d.ldy, d.tbl, ws, full)
        stretches, size = [], full
        while True:
            m.workspace_bytes = size
            F.fake_reset()
            if mx.lora_mx_linear(ctx, plan, m, 0, raw=True) != 0:
                break
            tile, = [g for n, g, _ in launched() if "mx_gemm" in n]
            stretches.append(tile[1])
            assert (tile[1] > 1) == any("splitk_reduce" in n for n, _, _ in launched())
            size -= one // 2
        assert stretches[0] > 1 and stretches[-1] == 1 and stretches == sorted(stretches, reverse=True), stretches
    """)
