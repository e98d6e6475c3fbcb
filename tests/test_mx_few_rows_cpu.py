"""include/lora_mx.h and its binding at the small end: every operator is a no-op for a batch without rows, whose tensors have no memory and
therefore null pointers; a single row may be cut out of a tensor of any stride."""
import pytest


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    import fake_hip
    return fake_hip.build(tmp_path_factory.mktemp("fake_hip"))


def test_no_rows(fake):
    import fake_hip
    fake_hip.run(fake, """
        import torch
        from paper_2505_14468_amd import mx
        K = 64
        x, g = torch.empty(0, K, dtype=torch.bfloat16), torch.ones(K, dtype=torch.bfloat16)
        assert x.data_ptr() == 0
        for h, y, q in ((x, x, "e4m3"), (None, x, None), (x, None, None), (None, None, "e4m3")):
            d = mx.norm_desc(x, g, 1e-5, residual=x if h is not None else None, h=h, y=y, q=mx.empty(0, K, q, "cpu") if q else None)
            assert mx.lora_rms_norm(ctx, d, 0, raw=True) == 0
        for fmt in ("e2m1", "e4m3"):
            d = mx.quantize_desc(x, mx.empty(0, K, fmt, "cpu"))
            assert mx.lora_mx_quantize(ctx, d, 0, raw=True) == mx.lora_mx_dequantize(ctx, d, 0, raw=True) == 0
        assert F.fake_launches() == 0
        plan = make_plan([0], [0], [8])
        F.fake_reset()
        for X8 in (None, mx.empty(0, K, "e4m3", "cpu")):
            W = mx.empty(40, K, "e2m1", "cpu")
            t = make_desc(plan, K, 40).tbl
            size = mx.lora_mx_linear_workspace_bytes(0, K, 40, 8, int(X8 is not None))
            rows = X8.struct if X8 is not None else mx.lora_mx_rows_t()
            d = mx.lora_mx_linear_desc(K, 40, 0, 0, None, K, rows, W.struct, None, 40, t, mem(size), size)
            assert mx.lora_mx_linear(ctx, plan, d, 0, raw=True) == 0 and mx.lora_mx_linear_multi(ctx, plan, [d, d], 0, raw=True) == 0
        assert F.fake_launches() == 0
        # with rows, an output is needed
        x = torch.zeros(2, K, dtype=torch.bfloat16)
        assert mx.lora_rms_norm(ctx, mx.norm_desc(x, g, 1e-5), 0, raw=True) == -1
    """)


def test_one_row_of_any_stride(fake):
    import fake_hip
    fake_hip.run(fake, """
        import torch
        from paper_2505_14468_amd import mx
        K = 64
        for dtype, wide in ((torch.bfloat16, 5004), (torch.float32, 5002)):
            cut = lambda n: torch.zeros(3, wide, dtype=dtype)[:1, :n]
            x, y, g = cut(K), cut(K), torch.ones(K, dtype=dtype)
            assert x.stride(0) == wide
            assert mx.lora_rms_norm(ctx, mx.norm_desc(x, g, 1e-5, residual=cut(K), h=cut(K), y=y, q=mx.empty(1, K, "e4m3", "cpu")), 0, raw=True) == 0
            q = mx.MxTensor(torch.zeros(3, 100, dtype=torch.uint8)[:1, :K], torch.zeros(3, 7, dtype=torch.uint8)[:1, :2], "e4m3")
            assert mx.lora_mx_quantize(ctx, mx.quantize_desc(x, q), 0, raw=True) == mx.lora_mx_dequantize(ctx, mx.dequantize_desc(q, y), 0, raw=True) == 0
        plan = make_plan([-1], [1], [8])
        class Pl:
            T, struct = 1, plan
        W = mx.empty(17, K, "e2m1", "cpu")
        ws = torch.zeros(mx.lora_mx_linear_workspace_bytes(1, K, 17, 8, 0) + 256, dtype=torch.uint8)
        ws = ws[-ws.data_ptr() % 256:]
        d = mx.linear_desc(Pl, torch.zeros(2, 5004, dtype=torch.bfloat16)[:1, :K], W, torch.zeros(2, 5004, dtype=torch.bfloat16)[:1, :17], None, ws)
        assert mx.lora_mx_linear(ctx, plan, d, 0, raw=True) == 0
    """)
