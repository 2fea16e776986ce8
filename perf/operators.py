"""Cases of the operators of a conditioned predictor block, as a user's program calls them through the Python binding.

Kinds:
  cross     attention of queries to an encoder's states of another length, ragged or masked
  quantize  rows as 8-bit floating point with a power-of-two scale for each block of 128 columns
  linear    activations quantized and multiplied with weights that were quantized once
  gnorm     group norm over channels-last positions with an activation

`own` picks between the plain forms (elementary torch operations in fp32) and the framework's kernels.
"""
import math

import torch

own = False

BLOCK = 128
LARGEST = 448.0                      # largest finite e4m3 value


def listed():
    cross = {"kind": "cross", "dtype": "bf16", "head_dim": 64, "heads": 30, "kv_heads": 30, "batch": 1, "ragged": False, "masked": False,
             "packed": False}
    return [
        # the 13 x 30 x 45 video tokens of the full network attend to its 226 text states, K and V halves of one projection
        dict(cross, name="cross_video_text", q_len=17550, kv_len=226, packed=True),
        # eight samples of one frame with prompts of their own lengths, padded to 226
        dict(cross, name="cross_padded_batch", batch=8, q_len=1350, kv_len=226, ragged=True),
        # 32 learned queries that pool all 17776 states, five query heads to a key head: few rows, a long axis
        dict(cross, name="cross_pool_long", batch=2, q_len=32, kv_len=17776, kv_heads=6),
        # a single token (a pooled embedding) against the text: nothing but latency
        dict(cross, name="cross_one_token", batch=2, q_len=1, kv_len=226, ragged=True),
        # a small fp32 network, 77 states with holes in the mask
        dict(cross, name="cross_f32_masked", batch=2, q_len=1000, kv_len=77, heads=16, kv_heads=16, head_dim=32, dtype="f32", masked=True),
        # the QKV projection of the full network: 17550 + 226 tokens
        {"name": "linear_qkv_full", "kind": "linear", "rows": 17776, "k": 1920, "n_out": 5760, "act": 0, "dtype": "bf16"},
        # the second MLP projection of one block on 4290 + 226 tokens
        {"name": "linear_fc2_block", "kind": "linear", "rows": 4516, "k": 7680, "n_out": 1920, "act": 0, "dtype": "bf16"},
        # the first MLP projection on the 112 tokens of a preview: weights are what is read
        {"name": "linear_fc1_few", "kind": "linear", "rows": 112, "k": 1920, "n_out": 7680, "act": 1, "dtype": "bf16"},
        # the MLP's activations of the full network
        {"name": "quantize_mlp_full", "kind": "quantize", "rows": 17776, "k": 7680, "dtype": "bf16"},
        # ragged fp32 rows that end inside a block
        {"name": "quantize_f32_ragged", "kind": "quantize", "rows": 333, "k": 1000, "dtype": "f32"},
        # 512 channels over the whole 13 x 60 x 90 latent
        {"name": "gnorm_latent", "kind": "gnorm", "batch": 1, "positions": 70200, "channels": 512, "groups": 32, "act": 2, "dtype": "bf16"},
        # a coarse level, fp32, groups of ten channels
        {"name": "gnorm_coarse", "kind": "gnorm", "batch": 2, "positions": 345, "channels": 320, "groups": 32, "act": 2, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["cross", "cross", "cross", "linear", "linear", "quantize", "gnorm", "gnorm"])
    while True:
        if kind == "cross":
            kv_heads = rng.choice([1, 2, 4, 6, 16, 30])
            c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]), "head_dim": rng.choice([16, 32, 64, 64, 64, 128]),
                 "kv_heads": kv_heads, "heads": kv_heads * rng.choice([1, 1, 5]), "batch": rng.choice([1, 1, 2, 3, 8]),
                 "q_len": _log(rng, 1, 17550), "kv_len": _log(rng, 1, 17776) if rng.random() < 0.4 else _log(rng, 16, 512),
                 "ragged": rng.random() < 0.4, "masked": rng.random() < 0.3, "packed": rng.random() < 0.3}
            c["masked"] = c["masked"] and c["kv_len"] >= 16          # (fewer keys could all be masked)
            scores = c["batch"] * c["heads"] * c["q_len"] * c["kv_len"]
            if scores <= 1.2e8 and scores * c["head_dim"] * (12 if c["dtype"] == "f32" else 1) <= 7.6e9:
                return c
        elif kind == "linear":
            c = {"kind": kind, "rows": _log(rng, 1, 17776), "k": _log(rng, 64, 7680), "n_out": 4 * _log(rng, 8, 1920), "act": rng.choice([0, 0, 1]),
                 "dtype": rng.choice(["bf16", "bf16", "f32"])}
            if work(c)["flops"] <= 3.9e11:
                return c
        elif kind == "quantize":
            c = {"kind": kind, "rows": _log(rng, 1, 17776), "k": _log(rng, 16, 7680), "dtype": rng.choice(["bf16", "f32"])}
            if work(c)["bytes"] <= 4.1e8:
                return c
        else:
            groups = rng.choice([1, 8, 32])
            c = {"kind": kind, "batch": rng.choice([1, 1, 2, 5]), "positions": _log(rng, 1, 70200), "groups": groups,
                 "channels": groups * 2 * _log(rng, 2, 1024 // groups), "act": rng.choice([0, 1, 2, 2]), "dtype": rng.choice(["bf16", "bf16", "f32"])}
            if work(c)["bytes"] <= 1.4e8:
                return c


def _type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def work(case):
    c = case
    if c["kind"] == "cross":
        size = 4 if c["dtype"] == "f32" else 2
        keys = c["kv_len"] * (0.6 if c["ragged"] else 1.0) * (0.8 if c["masked"] else 1.0)      # valid ones, on average
        return {"bytes": size * c["head_dim"] * c["batch"] * (2.0 * c["q_len"] * c["heads"] + 2.0 * keys * c["kv_heads"]),
                "flops": 4.0 * c["batch"] * c["heads"] * c["q_len"] * keys * c["head_dim"]}
    if c["kind"] == "linear":
        return {"bytes": c["rows"] * c["k"] * (4.0 if c["dtype"] == "f32" else 2.0) + 1.0 * c["n_out"] * c["k"] +
                c["rows"] * c["n_out"] * 2.0, "flops": 2.0 * c["rows"] * c["k"] * c["n_out"]}
    if c["kind"] == "quantize":
        return {"bytes": c["rows"] * c["k"] * ((4.0 if c["dtype"] == "f32" else 2.0) + 1.0), "flops": 3.0 * c["rows"] * c["k"]}
    n = c["batch"] * c["positions"] * c["channels"]
    return {"bytes": n * (8.0 if c["dtype"] == "f32" else 4.0), "flops": 10.0 * n}


def _quantize_plain(x):
    """Rows of x in blocks of 128 columns, the last one filled with zeros: (e4m3 values, e8m0 scales).  A block's scale is the least power
    of two under which its largest finite value is at most 448; what is not finite becomes NaN.  Scales lie block after block, one byte for
    each row, rows filled up to a multiple of 16 with the least scale."""
    rows, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    v = torch.zeros(rows, blocks * BLOCK, device=x.device)
    v[:, :cols] = x.float()
    v = v.view(rows, blocks, BLOCK)
    finite = torch.isfinite(v)
    mant, expo = torch.frexp(torch.where(finite, v.abs(), 0.0).amax(2))
    e = torch.where(mant > LARGEST / 512.0, expo - 8, expo - 9)          # 448 = 0.875 * 2^9
    e = torch.where(mant == 0, -127, e).clamp(-127, 127)
    y = torch.where(finite, v * torch.exp2(-e.float())[:, :, None], float("nan"))
    scale = torch.zeros(blocks, (rows + 15) // 16 * 16, dtype=torch.uint8, device=x.device)
    scale[:, :rows] = (e + 127).to(torch.uint8).t()
    return y.to(torch.float8_e4m3fn).view(rows, blocks * BLOCK), scale.view(torch.float8_e8m0fnu)


def _widen(q, scale):
    rows, cols = q.shape
    s = torch.exp2(scale.view(torch.uint8)[:, :rows].float() - 127.0)
    return (q.float().view(rows, -1, BLOCK) * s.t()[:, :, None]).view(rows, cols)


def prepare(case, seed):
    """Inputs on the GPU.  Matrices are N(0, 1/fan_in) and activations have channels of different size, so that outputs are of order one
    and block scales differ; what lies in keys that do not count is whatever an unwritten buffer holds, NaN among it."""
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _type(c["dtype"])
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    s = dict(c)
    if c["kind"] == "cross":
        b, nq, nk, h, hk, d = c["batch"], c["q_len"], c["kv_len"], c["heads"], c["kv_heads"], c["head_dim"]
        s["scale"] = 1.0 / math.sqrt(d)
        s["q"] = (1.5 * randn(b, nq, h, d)).to(dt)
        kv = randn(b, nk, 2, hk, d).to(dt)
        s["kv_lens"] = s["key_mask"] = None
        counts = torch.ones(b, nk, dtype=torch.bool, device="cuda")
        if c["ragged"]:
            s["kv_lens"] = (nk * (0.2 + 0.8 * rand(b))).ceil().to(torch.int32)
            counts &= torch.arange(nk, device="cuda") < s["kv_lens"][:, None]
        if c["masked"]:
            s["key_mask"] = rand(b, nk) < 0.8
            counts &= s["key_mask"]
        kv = torch.where(counts[:, :, None, None, None], kv, torch.full_like(kv, float("nan")))
        s["k"], s["v"] = (kv[:, :, 0], kv[:, :, 1]) if c["packed"] else (kv[:, :, 0].contiguous(), kv[:, :, 1].contiguous())
    elif c["kind"] in ("linear", "quantize"):
        s["x"] = (randn(c["rows"], c["k"]) * torch.exp(0.7 * randn(c["k"]))).to(dt)
        if c["kind"] == "linear":
            s["w"], s["w_scale"] = _quantize_plain(randn(c["n_out"], c["k"]) / math.sqrt(c["k"]))
            s["bias"] = randn(c["n_out"])
    else:
        ch = c["channels"]
        s["x"] = (randn(c["batch"], c["positions"], ch) * torch.exp(0.3 * randn(ch)) + 0.5 * randn(ch)).to(dt)
        s["gamma"], s["beta"] = 1.0 + 0.2 * randn(ch), 0.2 * randn(ch)
    return s


def _activate(x, act):
    if act == 1:
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    return x / (1.0 + torch.exp(-x)) if act == 2 else x


def _counted(s):
    b, nk = s["k"].shape[:2]
    m = torch.ones(b, nk, dtype=torch.bool, device=s["k"].device)
    if s["kv_lens"] is not None:
        m = m & (torch.arange(nk, device=m.device) < s["kv_lens"][:, None])
    return m if s["key_mask"] is None else m & s["key_mask"]


def _cross_plain(s):
    share = s["heads"] // s["kv_heads"]
    m = _counted(s)
    q = s["q"].float().permute(0, 2, 1, 3).contiguous()
    k, v = (torch.where(m[:, :, None, None], t.float(), 0.0).permute(0, 2, 1, 3).repeat_interleave(share, 1) for t in (s["k"], s["v"]))
    scores = s["scale"] * torch.matmul(q, k.transpose(2, 3).contiguous())
    out_of = ~m[:, None, None, :]
    top = scores.masked_fill(out_of, float("-inf")).amax(3, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), 0.0, top)).masked_fill(out_of, 0.0)
    total = p.sum(3, keepdim=True)
    o = torch.where(total > 0, torch.matmul(p, v) / total, 0.0)
    return o.permute(0, 2, 1, 3).contiguous().to(s["q"].dtype)


def _gnorm_plain(s):
    b, n, ch = s["x"].shape
    x = s["x"].float().view(b, n, s["groups"], ch // s["groups"])
    mean = x.mean((1, 3), keepdim=True)
    var = ((x - mean) ** 2).mean((1, 3), keepdim=True)
    y = ((x - mean) / torch.sqrt(var + 1e-5)).view(b, n, ch) * s["gamma"] + s["beta"]
    return _activate(y, s["act"]).to(s["x"].dtype)


def run(state):
    s = state
    kind = s["kind"]
    if own:
        from paper_2505_14741_amd import binding as B
        if kind == "cross":
            return B.cross_attn(s["q"], s["k"], s["v"], s["scale"], kv_lens=s["kv_lens"], key_mask=s["key_mask"])
        if kind == "quantize":
            return B.fp8_quantize(s["x"])
        if kind == "linear":
            a, a_scale = B.fp8_quantize(s["x"])
            return B.dit_linear_fp8(a, a_scale, s["w"], s["w_scale"], s["bias"], act=s["act"])
        return B.group_norm(s["x"], s["groups"], s["gamma"], s["beta"], eps=1e-5, act=s["act"])
    if kind == "cross":
        return _cross_plain(s)
    if kind == "quantize":
        return _quantize_plain(s["x"])
    if kind == "linear":
        y = torch.matmul(_widen(*_quantize_plain(s["x"])), _widen(s["w"], s["w_scale"]).t()) + s["bias"]
        return _activate(y, s["act"]).to(torch.bfloat16)
    return _gnorm_plain(s)


def _nearest_e4m3(y):
    """The e4m3 value next to each |y| <= 448 (ties to an even last bit): 3 bits behind the leading one, steps of 2^-9 below 2^-6."""
    _, x = torch.frexp(y.abs())
    step = torch.exp2((x - 1).clamp(min=-6).double() - 3.0)
    return torch.round(y / step) * step


def _exact_blocks(x):
    """fp64: values q and power-of-two scales s of x, block by block."""
    rows, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    v = torch.nn.functional.pad(x.double(), (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    top = v.abs().amax(2)
    e = torch.ceil(torch.log2(top / LARGEST).clamp(min=-127.0))
    for _ in range(2):                                   # (the logarithm may be off by its last bit next to a power of two)
        e = torch.where(top > LARGEST * torch.exp2(e), e + 1, e)
    e = torch.where((top <= LARGEST * torch.exp2(e - 1)) & (e > -127), e - 1, e)
    s = torch.exp2(e)
    return _nearest_e4m3(v / s[:, :, None]), s


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "cross":
        m = _counted(s)
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        share = s["heads"] // s["kv_heads"]
        o = torch.zeros_like(q)
        for b in range(s["batch"]):
            at = m[b].nonzero()[:, 0]
            for h in range(s["heads"]):
                if len(at):
                    z = (q[b, :, h] @ k[b, at, h // share].t()) * s["scale"]
                    z -= z.max(1, keepdim=True).values
                    w = z.exp_()
                    o[b, :, h] = (w @ v[b, at, h // share].contiguous()) / w.sum(1, keepdim=True)
        return o
    if kind == "gnorm":
        b, n, ch = s["x"].shape
        x = s["x"].double().view(b, n, s["groups"], -1)
        var, mean = torch.var_mean(x, (1, 3), correction=0, keepdim=True)
        y = ((x - mean) * torch.rsqrt(var + 1e-5)).reshape(b, n, ch) * s["gamma"].double() + s["beta"].double()
        return torch.nn.functional.gelu(y, approximate="tanh") if s["act"] == 1 else y * torch.sigmoid(y) if s["act"] == 2 else y
    q, e = _exact_blocks(s["x"])
    if kind == "quantize":
        fill = torch.full((q.shape[1], -q.shape[0] % 16), 2.0 ** -127, dtype=torch.float64, device=q.device)
        return q.reshape(q.shape[0], -1), torch.cat([e.t(), fill], 1)
    a = (q * e[:, :, None]).view(q.shape[0], -1)
    w = s["w"].double().view(s["w"].shape[0], -1, BLOCK)
    ws = torch.exp2(s["w_scale"].view(torch.uint8)[:, :w.shape[0]].double() - 127.0)
    y = a @ (w * ws.t()[:, :, None]).view(w.shape[0], -1).t() + s["bias"].double()
    return torch.nn.functional.gelu(y, approximate="tanh") if s["act"] else y
