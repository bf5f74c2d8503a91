"""Operators to measure: the 8-bit block-scaled matrix product, its activation quantiser, and the per-head
query/key norm with rotation and cache write.

Each case names its operator in "op":

  matmul   C = A B^T (+ add): E4M3 codes, one fp32 scale per row and 128 features of A, per 128 x 128 block of B
  quantize E4M3 codes and one fp32 scale per row and 128 features, of x or of silu(gate) * x
  qk       queries and keys normalised per head, rotated, and written (keys and values into a cache by slot)

With `own` false run() computes the plain form in elementary torch operations; with `own` true it calls the library.
"""
import math

import torch

own = False

GROUP = 128
E4M3_MAX = 448.0
AMAX_MIN = 2.0 ** -40  # the least maximum of a group
EPS = 1e-5
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one row's decode step: the fused q|k|v projection of the 8B shape
        dict(name="matmul_one_token", op="matmul", m=1, n=6144, k=4096, out="f16", add=False),
        # a decode step of a small group of rows: 8B down projection onto the residual stream
        dict(name="matmul_decode_group", op="matmul", m=24, n=4096, k=14336, out="f32", add=True),
        # the tiny model's down projection on a ragged batch: features that end inside a block
        dict(name="matmul_ragged", op="matmul", m=1021, n=256, k=688, out="bf16", add=False),
        # 8B output projection onto the residual stream, a mid-size batch
        dict(name="matmul_o_8b", op="matmul", m=2047, n=4096, k=4096, out="f32", add=True),
        # 1B gate|up projection, one batch of rows
        dict(name="matmul_gateup_1b", op="matmul", m=4093, n=16384, k=2048, out="f16", add=False),
        # 8B gate|up projection at the library's default batch of 16,384 tokens
        dict(name="matmul_gateup_8b", op="matmul", m=16384, n=28672, k=4096, out="f16", add=False),
        # one token's hidden state
        dict(name="quantize_one_token", op="quantize", rows=1, cols=4096, dtype="f16", gated=False),
        # a default batch's hidden states, 8B
        dict(name="quantize_hidden", op="quantize", rows=16384, cols=4096, dtype="f16", gated=False),
        # the MLP's middle, 8B, an odd number of tokens
        dict(name="quantize_gated", op="quantize", rows=4099, cols=14336, dtype="bf16", gated=True),
        # a decode step of nine rows, 8B heads, values into the library's transposed store
        dict(name="qk_decode_step", op="qk", tokens=9, heads=32, kv_heads=8, head_dim=128, dtype="f16",
             columns=True, slots=4096, holes=False),
        # a default batch, 8B heads
        dict(name="qk_prefill_8b", op="qk", tokens=16384, heads=32, kv_heads=8, head_dim=128, dtype="f16",
             columns=True, slots=16448, holes=False),
        # 1B heads, a cache of whole rows, padding tokens that write nothing
        dict(name="qk_rows_1b", op="qk", tokens=4093, heads=32, kv_heads=8, head_dim=64, dtype="bf16",
             columns=False, slots=8192, holes=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("matmul", "matmul", "quantize", "qk"))
    if op == "matmul":
        n, k = _log_int(rng, 64, 28672), _log_int(rng, 64, 14336)
        most = max(c["m"] * c["n"] * c["k"] for c in listed() if c["op"] == "matmul")
        m = _log_int(rng, 1, max(1, min(16384, most // (n * k))))
        out = rng.choice(("f16", "bf16", "f32"))
        return dict(op=op, m=m, n=n, k=k, out=out, add=out == "f32" and rng.random() < 0.5)
    if op == "quantize":
        return dict(op=op, rows=_log_int(rng, 1, 16384), cols=_log_int(rng, 64, 14336),
                    dtype=rng.choice(("f16", "bf16", "f32")), gated=rng.random() < 0.5)
    tokens = _log_int(rng, 1, 16384)
    kv_heads = rng.choice((1, 2, 4, 8))
    return dict(op=op, tokens=tokens, heads=kv_heads * rng.choice((1, 2, 3, 4, 7)), kv_heads=kv_heads,
                head_dim=rng.choice((64, 128)), dtype=rng.choice(("f16", "bf16")),
                columns=rng.random() < 0.5, slots=(tokens + rng.randrange(1, 512) + 7) // 8 * 8,
                holes=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs
def _up(x, to):
    return (x + to - 1) // to * to


def _groups(x):
    """x [rows][cols] padded with zeros to whole groups: [rows][groups][GROUP]."""
    pad = -x.shape[1] % GROUP
    x = torch.nn.functional.pad(x, (0, pad)) if pad else x
    return x.view(x.shape[0], -1, GROUP)


def _quantize(y):
    """Codes [rows][cols] and scales [rows][groups] of y in 32 bits."""
    g = _groups(y)
    amax = g.abs().amax(-1)
    bad = ~torch.isfinite(amax)
    amax = torch.where(bad, torch.full_like(amax, math.nan), amax.clamp(min=AMAX_MIN))
    q = (g * (E4M3_MAX / amax).unsqueeze(-1)).to(torch.float8_e4m3fn)
    return q.view(y.shape[0], -1)[:, :y.shape[1]], amax / E4M3_MAX


def _padded(q):
    """The same codes with rows a multiple of 16 bytes apart, as the product reads them."""
    out = torch.zeros(q.shape[0], _up(q.shape[1], 16), dtype=torch.uint8, device=q.device)
    out[:, :q.shape[1]] = q.view(torch.uint8)
    return out.view(torch.float8_e4m3fn)[:, :q.shape[1]]


def _quantize_blocks(w):
    """A weight's codes, with a scale for each 128 x 128 block."""
    n, k = w.shape
    p = torch.nn.functional.pad(w, (0, -k % GROUP, 0, -n % GROUP))
    b = p.view(p.shape[0] // GROUP, GROUP, -1, GROUP)
    amax = b.abs().amax((1, 3)).clamp(min=AMAX_MIN)
    q = (b * (E4M3_MAX / amax)[:, None, :, None]).to(torch.float8_e4m3fn).view(p.shape)
    return _padded(q[:n, :k]), (amax / E4M3_MAX).contiguous()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _hidden(rows, cols, g):
    """Hidden states: unit normal, a few features ten times as large."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    big = torch.rand(cols, generator=g, device="cuda") < 0.01
    return x * torch.where(big, 10.0, 1.0)


def _context(heads=1, kv_heads=1, head_dim=64):
    """The library's handle for this head layout (positions below 4096)."""
    from types import SimpleNamespace

    from paper_2606_31808_amd import lmop as L
    shape = SimpleNamespace(n_layers=0, d_model=64, n_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim,
                            d_ff=64, vocab=2, group_size=32, rms_eps=EPS, rope_theta=5e5)
    return L.Context(shape, device=torch.cuda.current_device(),
                     stream=torch.cuda.current_stream().cuda_stream, max_seq=4096)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        a, s["a_scale"] = _quantize(_hidden(m, k, g))
        s["a"] = _padded(a)
        s["b"], s["b_scale"] = _quantize_blocks(torch.randn(n, k, generator=g, device="cuda") * 0.02)
        s["residual"] = torch.randn(m, n, generator=g, device="cuda") if case["add"] else None
        if own:
            s["ctx"] = _context()
    elif case["op"] == "quantize":
        dt = DTYPES[case["dtype"]]
        s["x"] = _hidden(case["rows"], case["cols"], g).to(dt)
        s["gate"] = _hidden(case["rows"], case["cols"], g).to(dt) if case["gated"] else None
        if own:
            s["ctx"] = _context()
    else:
        T, nq, nkv, hd = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
        dt = DTYPES[case["dtype"]]
        # what a fused q|k|v projection leaves: one tensor, the three parts side by side
        s["qkv"] = (torch.randn(T, (nq + 2 * nkv) * hd, generator=g, device="cuda") * 2).to(dt)
        s["q_gain"], s["k_gain"] = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda") for _ in range(2))
        # rows of up to 96 tokens behind a prefix, one after the other in the cache
        start = int(torch.randint(0, 4000, (1,), generator=g, device="cuda"))
        s["pos"] = (start + torch.arange(T, device="cuda") % 96).to(torch.int32)
        first = int(torch.randint(0, case["slots"] - T + 1, (1,), generator=g, device="cuda"))
        slot = first + torch.arange(T, device="cuda")
        if case["holes"]:
            slot = torch.where(torch.rand(T, generator=g, device="cuda") < 0.1, -1, slot)
        s["slot"] = slot.to(torch.int32)
        s["k_store"] = torch.zeros(case["slots"], nkv * hd, dtype=dt, device="cuda")
        s["v_store"] = torch.zeros(*((nkv * hd, case["slots"]) if case["columns"] else (case["slots"], nkv * hd)),
                                   dtype=dt, device="cuda")
        if own:
            s["ctx"] = _context(nq, nkv, hd)
        else:
            angle = torch.arange(4096, device="cuda", dtype=torch.float64)[:, None] * _frequencies(hd)
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def _frequencies(hd):
    return 5e5 ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)


# ---------------------------------------------------------------- one pass
def run(s):
    return {"matmul": _run_matmul, "quantize": _run_quantize, "qk": _run_qk}[s["op"]](s)


def _run_matmul(s):
    if own:
        return s["ctx"].matmul(s["a"], s["a_scale"], s["b"], s["b_scale"], dtype=DTYPES[s["out"]], add=s["residual"])
    a = _groups(s["a"].float()) * s["a_scale"].unsqueeze(-1)
    b = _groups(s["b"].float()) * s["b_scale"].repeat_interleave(GROUP, 0)[:s["n"]].unsqueeze(-1)
    c = a.view(s["m"], -1) @ b.view(s["n"], -1).t()
    if s["residual"] is not None:
        c = c + s["residual"]
    return c.to(DTYPES[s["out"]])


def _run_quantize(s):
    if own:
        return s["ctx"].quantize(s["x"], gate=s["gate"])
    y = s["x"].float()
    if s["gate"] is not None:
        g = s["gate"].float()
        y = g / (1 + (-g).exp()) * y
    return _quantize(y)


def _run_qk(s):
    nq, nkv, hd = s["heads"], s["kv_heads"], s["head_dim"]
    q, k, v = s["qkv"].split((nq * hd, nkv * hd, nkv * hd), 1)
    if own:
        out = s["ctx"].qk_norm_rope(q, k, v, pos=s["pos"], q_gain=s["q_gain"], k_gain=s["k_gain"], slot=s["slot"],
                                    k_out=s["k_store"], v_out=s["v_store"], v_columns=s["columns"])
        return out, s["k_store"], s["v_store"]
    half = hd // 2
    cos, sin = (s[c][s["pos"].long()].unsqueeze(1) for c in ("cos", "sin"))

    def turned(x, gain):
        x = x.float().view(x.shape[0], -1, hd)
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        x1, x2 = x[..., :half], x[..., half:]
        return torch.cat((x1 * cos - x2 * sin, x1 * sin + x2 * cos), -1).view(x.shape[0], -1).to(s["qkv"].dtype)

    here = (s["slot"] >= 0).nonzero().squeeze(1) if s["holes"] else slice(None)
    at = s["slot"][here].long()
    s["k_store"][at] = turned(k, s["k_gain"])[here]
    if s["columns"]:
        s["v_store"][:, at] = v[here].t()
    else:
        s["v_store"][at] = v[here]
    return turned(q, s["q_gain"]), s["k_store"], s["v_store"]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = {"f16": 2, "bf16": 2, "f32": 4}
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        scales = 4 * (m * _up(k, GROUP) // GROUP + _up(n, GROUP) * _up(k, GROUP) // GROUP ** 2)
        return {"bytes": m * k + n * k + scales + m * n * (size[case["out"]] + (4 if case["add"] else 0)),
                "flops": 2.0 * m * n * k}
    if case["op"] == "quantize":
        e = case["rows"] * case["cols"]
        return {"bytes": e * (size[case["dtype"]] * (2 if case["gated"] else 1) + 1)
                + 4 * case["rows"] * (_up(case["cols"], GROUP) // GROUP), "flops": e * (10.0 if case["gated"] else 4.0)}
    e = case["tokens"] * (case["heads"] + 2 * case["kv_heads"]) * case["head_dim"]
    angles = 4.0 * case["tokens"] * case["head_dim"]
    return {"bytes": 2 * e * size[case["dtype"]] + 8 * case["tokens"] + angles, "flops": 7.0 * e}


# ---------------------------------------------------------------- the definition in 64 bits
def _e4m3(y):
    """The E4M3 value nearest to y (float64), ties to the even one: 3 fraction bits, least exponent -6."""
    e = torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4
    step = torch.pow(2.0, e.double())
    return (torch.round(y / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        feature = torch.arange(k, device="cuda") // GROUP
        row = torch.arange(n, device="cuda") // GROUP
        a = s["a"].double() * s["a_scale"].double()[:, feature]
        b = s["b"].double() * s["b_scale"].double()[row][:, feature]
        c = torch.mm(a, b.t().contiguous())
        return c + s["residual"].double() if case["add"] else c
    if case["op"] == "quantize":
        y = s["x"].double()
        if case["gated"]:
            y = torch.sigmoid(s["gate"].double()) * s["gate"].double() * y
        cols, groups = case["cols"], _up(case["cols"], GROUP) // GROUP
        top = torch.full((case["rows"], groups), AMAX_MIN, dtype=torch.float64, device="cuda")
        group = (torch.arange(cols, device="cuda") // GROUP).expand(case["rows"], cols)
        top.scatter_reduce_(1, group, y.abs(), "amax")
        return _e4m3(y * E4M3_MAX / top.gather(1, group)), top / E4M3_MAX
    T, nq, nkv, hd = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    x = s["qkv"].double().view(T, nq + 2 * nkv, hd)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["pos"].double()[:, None, None] * _frequencies(hd))

    def heads(x, gain):
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gain.double()
        z = torch.complex(x[..., :hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * turn
        return torch.cat((z.real, z.imag), -1).reshape(T, -1)

    k_store, v_store = s["k_store"].double(), s["v_store"].double()
    live = s["slot"] >= 0
    at = s["slot"][live].long()
    k_store[at] = heads(x[:, nq:nq + nkv], s["k_gain"])[live]
    v = x[:, nq + nkv:].reshape(T, -1)[live]
    if case["columns"]:
        v_store[:, at] = v.t()
    else:
        v_store[at] = v
    return heads(x[:, :nq], s["q_gain"]), k_store, v_store
