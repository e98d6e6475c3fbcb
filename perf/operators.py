"""The work that the operators of a 4-bit backbone are measured on: the multi-LoRA linear layer whose backbone weights are
held in 4 bits with a scale for every 32 of them, the root-mean-square norm in front of it, whose output comes in 8 bits with
scales as well, and the conversions in and out of both formats.

Formats: blocks of 32 consecutive values along a row share a scale 2^(s - 127), s one byte; the values are held as e2m1 (4
bits, two a byte, the even one in the low half) or as e4m3 (8 bits).  The scale of a block is the smallest power of two with
which its largest value stays in the format's range (6 or 448); values are rounded to nearest, ties to even.

``run`` with ``own`` false computes everything from elementary torch operations in fp32; with ``own`` true it calls the
library on descriptors that the program made once, as a serving loop does.  What is held in 8 or 4 bits is returned as the
values it stands for (bf16 holds them exactly), which is a conversion of its own on either side.
"""
import numpy as np
import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def _norm(name, rows, K, dtype="bf16", residual=True, quantized=True):
    return dict(name=name, op="norm", rows=rows, K=K, dtype=dtype, residual=residual, quantized=quantized)


def _quantize(name, rows, K, fmt, dtype="bf16"):
    return dict(name=name, op="quantize", rows=rows, K=K, fmt=fmt, dtype=dtype)


def _linear(name, K, N, requests, length, mean, sets=1, x8=False, adapters=1, ids="uniform", ranks="16", bare=0.0, mix=1):
    """length: "one" (a token a request), "fixed" (`mean` tokens), "uniform" (mean/4 .. 7/4 mean), "mixed" (four prefills of `mean`
    tokens among one-token requests).  ids: "uniform" or "zipf".  ranks: one drawn per adapter.  adapters 0: the backbone alone."""
    return dict(name=name, op="linear", K=K, N=N, sets=sets, x8=x8, requests=requests, length=length, mean=mean, adapters=adapters,
                ids=ids, ranks=ranks, bare=bare, mix=mix)


def listed():
    return [
        # one user, one token: the latency of a norm in a decode step
        _norm("norm_one", 1, 4096, quantized=False),
        # an ordinary decode batch in front of q/k/v
        _norm("norm_73", 73, 4096),
        # a prefill batch in front of gate/up
        _norm("norm_7500", 7500, 4096),
        # full precision, the wide side of an MLP, no residual (a norm inside a block)
        _norm("norm_f32_391", 391, 11008, dtype="f32", residual=False, quantized=False),
        # an up projection's weights on their way into 4 bits, when a model is loaded
        _quantize("quantize_weights", 11008, 4096, "e2m1"),
        # the input of a down projection, which no norm precedes
        _quantize("quantize_rows", 391, 11008, "e4m3"),
        # one user, one token, one projection: weights streamed, latency
        _linear("linear_one", 4096, 4096, 1, "one", 1, adapters=32),
        # an ordinary decode batch through an up projection
        _linear("linear_64_up", 4096, 11008, 64, "one", 1, adapters=32),
        # a decode batch through q/k/v of a 7B layer in one call, inputs in 8 bits as the norm leaves them, mixed ranks
        _linear("linear_73_qkv_x8", 4096, 4096, 73, "one", 1, sets=3, x8=True, adapters=100, ranks="8,16,32,64", bare=0.1),
        # a few hundred ragged rows (short prompts) through a down projection, inputs in 16 bits
        _linear("linear_391_down", 11008, 4096, 23, "uniform", 17, adapters=16, ranks="16,32", bare=0.1),
        # decode requests with a few prefills among them, inputs in 8 bits
        _linear("linear_1216_up_x8", 4096, 11008, 196, "mixed", 256, x8=True, adapters=100, ranks="8,16,32,64"),
        # a prefill batch through an up projection, ragged lengths, few adapters, inputs in 8 bits
        _linear("linear_7500_up_x8", 4096, 11008, 13, "uniform", 577, x8=True, adapters=8, ids="zipf", ranks="64"),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def log_int(lo, hi):
        return int(round(2.0 ** rng.uniform(np.log2(lo), np.log2(hi))))

    op = rng.choice(["norm", "quantize", "linear", "linear", "linear"])
    if op == "norm":
        rows, K = log_int(1, 7500), 32 * log_int(8, 512)
        while rows * K > 7500 * 4096:
            rows = rows * 2 // 3
        c = _norm("", rows, K, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.7, rng.random() < 0.6)
    elif op == "quantize":
        rows, K = log_int(1, 13824), 32 * log_int(8, 432)
        while rows * K > 11008 * 4096:
            rows = rows * 2 // 3
        c = _quantize("", rows, K, rng.choice(["e2m1", "e4m3"]), rng.choice(["bf16", "bf16", "f32"]))
    else:
        length = rng.choice(["one", "one", "uniform", "mixed"])
        if length == "one":
            requests, mean = log_int(1, 1500), 1
        elif length == "mixed":
            requests, mean = log_int(8, 256), log_int(16, 280)
        else:
            requests = log_int(1, 24)
            mean = log_int(8, max(9, int(7500 / 1.75 / requests)))
        K, N = rng.choice([(4096, 4096), (4096, 11008), (11008, 4096), (5120, 5120), (5120, 13824),
                           (32 * log_int(8, 344), log_int(200, 12288)), (32 * log_int(8, 344), log_int(200, 12288))])
        c = _linear("", K, N, requests, length, mean, x8=rng.random() < 0.5, adapters=rng.choice([0, log_int(1, 128), log_int(1, 128)]),
                    ids=rng.choice(["uniform", "zipf"]), ranks=rng.choice(["8", "16", "64", "16,32", "8,16,32,64"]),
                    bare=rng.choice([0.0, 0.1, 0.3]), mix=rng.randrange(1 << 30))
        rows = int(_geometry(c)[1].sum())
        if rows * K * N > 4500 * 4096 * 11008:
            c["K"], c["N"] = 4096, 4096
        elif rows <= 128:
            c["sets"] = rng.choice([1, 1, 2, 3])
    del c["name"]
    return c


def _geometry(case):
    """Adapter id and token count of every request, rank of every adapter: from the case alone."""
    rng = np.random.default_rng([7, case["mix"]])
    n, mean, pool = case["requests"], case["mean"], case["adapters"]
    if case["length"] == "uniform":
        ntok = rng.integers(max(1, mean // 4), max(2, mean * 7 // 4 + 1), n)
    elif case["length"] == "mixed":
        ntok = np.where(np.arange(n) < 4, mean, 1)
    else:
        ntok = np.full(n, mean)
    if pool == 0:
        return np.full(n, -1, np.int32), ntok.astype(np.int32), np.zeros(0, np.int32)
    if case["ids"] == "zipf":
        w = 1.0 / np.arange(1, pool + 1)
        ids = rng.choice(pool, n, p=w / w.sum())
    else:
        ids = rng.integers(0, pool, n)
    ids = np.where(rng.random(n) < case["bare"], -1, ids)
    ranks = rng.choice([int(r) for r in case["ranks"].split(",")], pool)
    return ids.astype(np.int32), ntok.astype(np.int32), ranks.astype(np.int32)


# ---- the formats, in elementary operations -----------------------------------------------------------------------------

def _scale_exponent(v, fmt):
    """Exponent of the block scales of `v` ([rows, K], fp32), [rows, K / 32]: largest value <= limit * 2^e."""
    amax = v.view(v.shape[0], -1, 32).abs().amax(-1)
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1); the limits are 0.75 * 2^3 and 0.875 * 2^9
    top, shift = (0.75, 3) if fmt == "e2m1" else (0.875, 9)
    e = e - shift + (m > top).to(e.dtype)
    return torch.where(amax > 0, e, -127).clamp(-127, 127)


def _round_e2m1(a):
    """Magnitudes up to 6 to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code."""
    half = (a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float()
    return 0.5 * half + (a > 2.5).float() + (a >= 3.5).float() + 2.0 * (a > 5.0).float()


def _parts(v, fmt):
    """(rounded values of the format, scale exponents) of `v` in fp32."""
    e = _scale_exponent(v, fmt)
    u = torch.ldexp(v.view(v.shape[0], -1, 32), -e.unsqueeze(-1)).view(v.shape)
    if fmt == "e2m1":
        return torch.copysign(_round_e2m1(u.abs()), u), e
    return u.to(torch.float8_e4m3fn).float(), e


def _values(u, e):
    """What rounded values and scale exponents stand for, in fp32."""
    return torch.ldexp(u.view(u.shape[0], -1, 32), e.unsqueeze(-1)).view(u.shape)


def _held(v, fmt):
    """(codes, scales) as bytes, as a checkpoint holds them."""
    u, e = _parts(v, fmt)
    scales = (e + 127).to(torch.uint8)
    if fmt == "e4m3":
        return u.to(torch.float8_e4m3fn).view(torch.uint8), scales
    a = u.abs()
    code = (torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)) + 8 * torch.signbit(u)).to(torch.uint8)
    return (code[:, 0::2] | code[:, 1::2] << 4).contiguous(), scales


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _opened(codes, scales, fmt):
    """fp32 values of codes and scales."""
    if fmt == "e4m3":
        u = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(_E2M1, device=codes.device)
        u = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).view(codes.shape[0], -1)
    return _values(u, scales.int() - 127)


# ---- inputs --------------------------------------------------------------------------------------------------------------

_context = None


def _ctx():
    """One library context per process, as a program keeps it."""
    global _context
    if _context is None:
        from paper_2505_14468_amd import runtime as rt
        _context = rt.Context(0)
    return _context


def _normal(gen, rows, cols, sigma=1.0, dtype=torch.bfloat16):
    return torch.randn((rows, cols), generator=gen, device=DEVICE, dtype=dtype).mul_(sigma)


def _hidden(gen, rows, K, dtype=torch.bfloat16):
    """A residual stream: a few of its channels are some twenty times as large as the rest."""
    x = _normal(gen, rows, K, dtype=dtype)
    loud = torch.randint(K, (max(1, K // 512),), generator=gen, device=DEVICE)
    x[:, loud] *= 20.0
    return x


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    state = dict(case, dtype=DTYPES[case.get("dtype", "bf16")])
    if case["op"] == "norm":
        state["x"] = _hidden(gen, case["rows"], case["K"], state["dtype"])
        state["r"] = _hidden(gen, case["rows"], case["K"], state["dtype"]) if case["residual"] else None
        state["g"] = (1.0 + 0.2 * torch.randn(case["K"], generator=gen, device=DEVICE)).to(state["dtype"])
    elif case["op"] == "quantize":
        make = _normal if case["fmt"] == "e2m1" else _hidden
        state["x"] = make(gen, case["rows"], case["K"], dtype=state["dtype"])
        if case["fmt"] == "e2m1":
            state["x"].mul_(0.02)
    else:
        K, N = case["K"], case["N"]
        ids, ntok, ranks = _geometry(case)
        order = np.random.default_rng([11, seed]).permutation(len(ids))
        ids, ntok = np.ascontiguousarray(ids[order]), np.ascontiguousarray(ntok[order])
        state.update(ids=ids, ntok=ntok, ranks=ranks)
        state["X"] = _hidden(gen, int(ntok.sum()), K)
        state["X8"] = _held(state["X"].float(), "e4m3") if case["x8"] else None
        # of every projection: the backbone's codes and scales, the adapters' weights one after the other along the ranks
        state["W"] = [_held(_normal(gen, N, K, 0.02).float(), "e2m1") for _ in range(case["sets"])]
        R = int(ranks.sum())
        state["A"] = [_normal(gen, R, K, K ** -0.5) for _ in range(case["sets"])]
        state["B"] = [_normal(gen, N, R, 0.02) for _ in range(case["sets"])]
        state["scale"] = (16.0 / ranks).astype(np.float32)
        # adapter of every row, and of every column of the ranks
        state["row_adapter"] = torch.from_numpy(np.repeat(ids, ntok)).to(DEVICE)
        state["col_adapter"] = torch.from_numpy(np.repeat(np.arange(len(ranks)), ranks).astype(np.int32)).to(DEVICE)
        state["col_scale"] = torch.from_numpy(np.repeat(state["scale"], ranks)).to(DEVICE)
    if own:
        _keep(state)
    return state


def _keep(s):
    """What a serving loop makes once and keeps: descriptors with their outputs, and for the linear layer the batch's plan, the
    adapter tables and the workspaces."""
    from paper_2505_14468_amd import mx
    from paper_2505_14468_amd import runtime as rt
    ctx = s["ctx"] = _ctx()
    if s["op"] == "norm":
        rows, K = s["x"].shape
        s["y"] = torch.empty_like(s["x"])
        s["h"] = torch.empty_like(s["x"]) if s["residual"] else None
        s["q"] = mx.empty(rows, K, "e4m3", ctx.device) if s["quantized"] else None
        s["desc"] = mx.norm_desc(s["x"], s["g"], EPS, residual=s["r"], h=s["h"], y=s["y"], q=s["q"])
    elif s["op"] == "quantize":
        s["q"] = mx.empty(*s["x"].shape, s["fmt"], ctx.device)
        s["desc"] = mx.quantize_desc(s["x"], s["q"])
    else:
        T, N = s["X"].shape[0], s["N"]
        s["plan"] = rt.plan(ctx, s["ids"], s["ntok"], s["ranks"])
        X8 = mx.MxTensor(*s["X8"], "e4m3") if s["x8"] else None
        at = np.concatenate([[0], np.cumsum(s["ranks"])]).astype(int)
        s["held"], s["descs"], s["out"] = [X8], [], []
        for (codes, scales), A, Bw in zip(s["W"], s["A"], s["B"]):
            table = None
            if len(s["ranks"]):
                table = rt.AdapterTable([A[i:j] for i, j in zip(at, at[1:])], [Bw[:, i:j].contiguous() for i, j in zip(at, at[1:])],
                                        s["scale"], ctx.device)
            W = mx.MxTensor(codes, scales, "e2m1")
            Y = torch.empty((T, (N + 7) // 8 * 8), dtype=torch.bfloat16, device=ctx.device)[:, :N]
            ws = mx.workspace(T, s["K"], N, s["plan"].r_max, ctx.device, x8=s["x8"])
            s["descs"].append(mx.linear_desc(s["plan"], s["X"], W, Y, table, ws, X8))
            s["held"] += [W, table, ws]
            s["out"].append(Y)
    if s.get("q") is not None:
        s["v"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device=ctx.device)
        s["vdesc"] = mx.dequantize_desc(s["q"], s["v"])


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "norm":
        h = s["x"].float()
        if s["residual"]:
            h = h + s["r"].float()
        y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["g"].float()
        out = {"y": y.to(s["dtype"])}
        if s["residual"]:
            out["h"] = h.to(s["dtype"])
        if s["quantized"]:
            out["v"] = _values(*_parts(y, "e4m3")).bfloat16()
        return out
    if s["op"] == "quantize":
        return _values(*_parts(s["x"].float(), s["fmt"])).bfloat16()
    X = s["X"].float()
    Xb = _opened(*s["X8"], "e4m3") if s["x8"] else X
    mine = (s["row_adapter"][:, None] == s["col_adapter"][None, :]) * s["col_scale"]
    return [(Xb @ _opened(*W, "e2m1").t() + ((X @ A.float().t()) * mine) @ Bw.float().t()).bfloat16()
            for W, A, Bw in zip(s["W"], s["A"], s["B"])]


def _run_own(s):
    from paper_2505_14468_amd import mx
    ctx, stream = s["ctx"], torch.cuda.current_stream().cuda_stream
    if s["op"] == "norm":
        mx.lora_rms_norm(ctx.handle, s["desc"], stream)
        out = {"y": s["y"]}
        if s["residual"]:
            out["h"] = s["h"]
        if s["quantized"]:
            mx.lora_mx_dequantize(ctx.handle, s["vdesc"], stream)
            out["v"] = s["v"]
        return out
    if s["op"] == "quantize":
        mx.lora_mx_quantize(ctx.handle, s["desc"], stream)
        mx.lora_mx_dequantize(ctx.handle, s["vdesc"], stream)
        return s["v"]
    if len(s["descs"]) == 1:
        mx.lora_mx_linear(ctx.handle, s["plan"].struct, s["descs"][0], stream)
    else:
        mx.lora_mx_linear_multi(ctx.handle, s["plan"].struct, s["descs"], stream)
    return s["out"]


def work(case):
    if case["op"] != "linear":
        n, es = case["rows"] * case["K"], 2 if case["dtype"] == "bf16" else 4
        if case["op"] == "quantize":  # in, codes and scales out; those in, 16-bit values out
            held = n * (0.5 if case["fmt"] == "e2m1" else 1.0) + n / 32
            return {"bytes": n * es + 2 * held + 2 * n, "flops": 4 * n}
        nbytes = n * es * (4 if case["residual"] else 2) + case["K"] * es
        if case["quantized"]:
            nbytes += 2 * (n + n / 32) + 2 * n
        return {"bytes": nbytes, "flops": 5 * n}
    ids, ntok, ranks = _geometry(case)
    T, K, N, sets = int(ntok.sum()), case["K"], case["N"], case["sets"]
    used = np.unique(ids[ids >= 0])
    r_used = int(ranks[used].sum())
    r_rows = int((np.where(ids >= 0, ranks[np.maximum(ids, 0)], 0) * ntok).sum()) if len(ranks) else 0
    nbytes = (T * K * 33 / 32 if case["x8"] else 0) + (2 * T * K if not case["x8"] or r_used else 0)
    nbytes += sets * (N * K / 2 + N * K / 32 + 2 * T * N + 2 * r_used * (K + N))
    return {"bytes": nbytes, "flops": sets * (2 * T * K * N + 2 * r_rows * (K + N))}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------

def _exact_held(v, fmt):
    """What is held of `v` (64 bits): every value the nearest multiple of its step, the step from its own exponent."""
    top, mantissa, lowest = (6.0, 1, 0) if fmt == "e2m1" else (448.0, 3, -6)
    v = v.view(v.shape[0], -1, 32)
    limit = v.abs().amax(-1, keepdim=True) / top
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(limit > 0, limit, torch.ones_like(limit)))))
    scale = torch.where(limit > scale, 2 * scale, torch.where(limit <= scale / 2, scale / 2, scale)).clamp(2.0 ** -127, 2.0 ** 127)
    u = v / scale
    exponent = torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -60))).clamp_min(lowest)
    step = torch.exp2(exponent - mantissa)
    return (torch.round(u / step) * step * scale).flatten(1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].double() + (s["r"].double() if case["residual"] else 0.0)
        y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + EPS) * s["g"].double()
        out = {"y": y}
        if case["residual"]:
            out["h"] = h
        if case["quantized"]:
            out["v"] = _exact_held(y, "e4m3")
        return out
    if case["op"] == "quantize":
        return _exact_held(s["x"].double(), case["fmt"])
    X = s["X"].double()
    block = lambda e: torch.exp2(e.double() - 127).repeat_interleave(32, 1)  # noqa: E731
    Xb = X if not case["x8"] else s["X8"][0].view(torch.float8_e4m3fn).double() * block(s["X8"][1])
    at = np.concatenate([[0], np.cumsum(s["ranks"])]).astype(int)
    outs = []
    for (codes, scales), A, Bw in zip(s["W"], s["A"], s["B"]):
        W = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
        for half, code in ((0, codes & 15), (1, codes >> 4)):
            m, e = (code & 1).double(), ((code >> 1) & 3).double()
            W[:, half::2] = torch.where(e > 0, (1 + m / 2) * torch.exp2(e - 1), m / 2) * (1 - 2 * (code >> 3).double())
        Y = Xb @ (W * block(scales)).t()
        for a in np.unique(s["ids"][s["ids"] >= 0]):
            rows = torch.nonzero(s["row_adapter"] == int(a)).flatten()
            i, j = at[a], at[a + 1]
            Y[rows] += float(s["scale"][a]) * ((X[rows] @ A[i:j].double().t()) @ Bw[:, i:j].double().t())
        outs.append(Y)
    return outs
