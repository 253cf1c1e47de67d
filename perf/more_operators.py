"""Experts in microscaled 4 bits (MX4: e2m1 values, one power-of-two scale per 32
columns), as measurable cases: each is one pass through an operator on inputs that
are already on the GPU.

  quant    moe_mx4_quantize and moe_mx4_dequantize: the codes and scales of a matrix,
           and what they stand for
  product  moe_mx4_grouped_product: the routed rows (MX4 or bf16) times each expert's
           MX4 matrix
  ffn      moe_grouped_ffn_fwd_mx4: the SwiGLU experts at MX4 weights, activations in
           MX4 (act 4) or in bf16 (act 16), tokens gathered by the routing

Sizes are the repository's layers (d_model 1024, 2048 and 4096, d_ff 1024 and 2048,
64 experts top-8 and top-2, 45 of 64 after pruning), from a single token to 8192.
Values: normalised tokens with a few large channels, weights ~ N(0, 0.02), routing by
logits with a skewed bias.

With ``own`` false the operators are computed from their formulas by elementary
torch operations in float32, each output rounded once.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32          # columns that share a scale
GROUP = 256         # columns whose eight scales lie together: scale [C / 256, R, 8]


def listed():
    return [
        # the normalised tokens of eight sequences decoding, one token each: latency
        dict(name="quant_decode_8", kind="quant", n=1, R=8, C=2048, dtype="bf16"),
        # one prompt of odd length, fp32, columns that fill no whole group of scales
        dict(name="quant_1531_f32", kind="quant", n=1, R=1531, C=1056, dtype="f32"),
        # the down projections of the `balanced` layer's 64 experts, when a model is loaded
        dict(name="quant_experts", kind="quant", n=64, R=2048, C=1024, dtype="bf16"),
        # one dense projection (a single expert) of eight decoding tokens
        dict(name="product_decode_8", kind="product", T=8, k=1, E=1, dead=0, N=2048, K=2048,
             act=4, dtype="bf16"),
        # odd sizes in float32 out: a prompt over the 45 experts left of 64, uneven loads
        dict(name="product_1531_f32", kind="product", T=1531, k=2, E=64, dead=19, N=1088, K=1216,
             act=16, dtype="f32"),
        # the `balanced` layer's gate/up product: 8192 tokens x 8 slots
        dict(name="product_balanced", kind="product", T=8192, k=8, E=64, dead=0, N=2048, K=2048,
             act=4, dtype="bf16"),
        # a single token decoding: eight experts' weights
        dict(name="ffn4_decode_1", kind="ffn", T=1, k=8, E=64, dead=0, d=2048, f=1024, act=4),
        # sixteen sequences decoding through the pruned layer, activations in bf16
        dict(name="ffn16_decode_16", kind="ffn", T=16, k=8, E=64, dead=19, d=2048, f=1024, act=16),
        # a short prompt of odd length through the wide top-2 layer
        dict(name="ffn4_1531", kind="ffn", T=1531, k=2, E=16, dead=0, d=4096, f=2048, act=4),
        # a chunk of a prompt, activations in bf16
        dict(name="ffn16_1024", kind="ffn", T=1024, k=8, E=64, dead=0, d=2048, f=1024, act=16),
        # the `balanced` layer, 8192 tokens
        dict(name="ffn4_balanced", kind="ffn", T=8192, k=8, E=64, dead=0, d=2048, f=1024, act=4),
        dict(name="ffn16_balanced", kind="ffn", T=8192, k=8, E=64, dead=0, d=2048, f=1024, act=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, hi):
    return 64 * rng.choice([rng.randint(1, hi // 64), 2 ** rng.randint(0, (hi // 64).bit_length() - 1)])


def draw(rng):
    kind = rng.choice(["quant", "product", "product", "ffn", "ffn", "ffn"])
    if kind == "quant":
        C = 32 * rng.choice([rng.randint(1, 128), 2 ** rng.randint(1, 7)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 64 * 2048 * 1024 // (1 if dtype == "bf16" else 2)
        n = rng.choice([1, 1, rng.randint(2, 16)])
        return dict(kind=kind, n=n, R=_log(rng, 1, min(131072, most // (C * n))), C=C, dtype=dtype)
    E = rng.choice([1, 8, 16, 64, 64, rng.randint(2, 128)])
    dead = rng.choice([0, 0, E // 4])
    k = rng.choice([k for k in (1, 2, 4, 8) if k <= E - dead])
    a, b = _width(rng, 4096), _width(rng, 2048)
    while E * a * b > 64 * 2048 * 1024:          # the listed layers' weights
        E = max(1, E // 2)
        dead, k = 0, min(k, E)
    T = _log(rng, 1, min(8192, 8192 * 8 * 2048 * 1024 // (k * a * b)))
    act = rng.choice([4, 4, 16])
    if kind == "product":
        a, b = (a, b) if rng.random() < 0.5 else (b, a)
        return dict(kind=kind, T=T, k=k, E=E, dead=dead, N=a, K=b, act=act,
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    return dict(kind=kind, T=T, k=k, E=E, dead=dead, d=a, f=b, act=act)


# ---------------------------------------------------------------------------------------
# inputs, from the seed alone
# ---------------------------------------------------------------------------------------
def _normal(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g)


def _tokens(g, T, d):
    """Normalised tokens: unit rows, a few channels much larger."""
    scale = torch.exp(_normal(g, d, std=0.4))
    scale[torch.randint(0, d, (max(1, d // 256),), device=DEV, generator=g)] *= 8.0
    return _normal(g, T, d) * scale


def _weights(g, n, N, K):
    """The experts' MX4 matrices, as a program holds them: codes and scales."""
    return _plain_quantize(_normal(g, n, N, K, std=0.02).to(torch.bfloat16))


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]
    if kind == "quant":
        n, R, C = case["n"], case["R"], case["C"]
        if n == 1:
            return dict(src=_tokens(g, R, C).to(DTYPES[case["dtype"]]))
        return dict(src=_normal(g, n, R, C, std=0.02).to(DTYPES[case["dtype"]]))
    T, k, E, dead = case["T"], case["k"], case["E"], case["dead"]
    logits = _normal(g, T, E) + _normal(g, E, std=0.7)
    gone = torch.randperm(E, device=DEV, generator=g)[:dead]
    logits[:, gone] = -math.inf
    idx = torch.topk(logits, k, dim=1).indices
    # the dispatch as moe_expert_counts leaves it: routed rows by expert, then by token
    flat = idx.reshape(-1)
    row_src = torch.sort(flat, stable=True).indices
    counts = torch.zeros(E, dtype=torch.int64, device=DEV).index_add_(
        0, flat, torch.ones_like(flat))
    alive = torch.ones(E, dtype=torch.int64, device=DEV)
    alive[gone] = 0
    slot = torch.where(alive > 0, torch.cumsum(alive, 0) - 1, torch.full_like(alive, -1))
    v = dict(row_src=row_src.to(torch.int32),
             offsets=torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)]).to(torch.int32),
             expert_map=slot.to(torch.int32) if dead else None)
    v["cap"] = int(counts.max())          # rows of the fullest expert
    if kind == "product":
        x = _tokens(g, T, case["K"])
        v["x"] = _plain_quantize(x) if case["act"] == 4 else x.to(torch.bfloat16)
        v["w"] = _weights(g, E - dead, case["N"], case["K"])
    else:
        v["x"] = _tokens(g, T, case["d"]).to(torch.bfloat16)
        v["w_gate_up"] = _weights(g, E - dead, 2 * case["f"], case["d"])
        v["w_down"] = _weights(g, E - dead, case["d"], case["f"])
    return v


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    if own:
        state["out"] = _buffers(case, state)
    return state


def _buffers(case, v):
    """The output buffers and workspaces that a program keeps from call to call."""
    import paper_2601_14327_amd as laep

    if case["kind"] == "quant":
        s = v["src"]
        codes = torch.empty(s.shape[:-1] + (s.shape[-1] // 2,), dtype=torch.uint8, device=DEV)
        scale = torch.empty(s.shape[:-2] + (-(-s.shape[-1] // GROUP), s.shape[-2], 8),
                            dtype=torch.uint8, device=DEV)
        return dict(codes=codes, scale=scale), torch.empty_like(s)
    T, k, E = case["T"], case["k"], case["E"]
    if case["kind"] == "product":
        nbytes = laep.workspace_bytes(laep.LAEP_CALL_MX4_PRODUCT, T, k, E, case["K"], case["N"])
        out = torch.empty((T * k, case["N"]), dtype=DTYPES[case["dtype"]], device=DEV)
        return dict(out=out, ws=torch.empty(max(nbytes, 1), dtype=torch.uint8, device=DEV))
    nbytes = laep.workspace_bytes(laep.LAEP_CALL_MX4_FFN, T, k, E, case["d"], case["f"])
    return dict(y_perm=torch.empty((T * k, case["d"]), dtype=torch.bfloat16, device=DEV),
                ws=torch.empty(max(nbytes, 1), dtype=torch.uint8, device=DEV))


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(v):
    import paper_2601_14327_amd as laep

    c = v["case"]
    if c["kind"] == "quant":
        kept, out = v["out"]
        codes, scale = laep.moe_mx4_quantize(v["src"], **kept)
        return laep.moe_mx4_dequantize(codes, scale, v["src"].dtype, out=out)
    if c["kind"] == "product":
        x = laep.Mx4(*v["x"]) if c["act"] == 4 else v["x"]
        return laep.moe_mx4_grouped_product(x, laep.Mx4(*v["w"]), v["offsets"],
                                            row_src=v["row_src"], k=c["k"],
                                            expert_map=v["expert_map"], dtype=DTYPES[c["dtype"]],
                                            **v["out"])
    y, _ = laep.moe_grouped_ffn_fwd_mx4(v["x"], laep.Mx4(*v["w_gate_up"]), laep.Mx4(*v["w_down"]),
                                        v["offsets"], row_src=v["row_src"], k=c["k"],
                                        act_bits=c["act"], expert_map=v["expert_map"], **v["out"])
    return y


def _plain_quantize(x):
    """codes [..., R, C / 2] (even columns in the low halves) and scales
    [..., ceil(C / 256), R, 8], biased exponents."""
    C = x.shape[-1]
    v = x.float().unflatten(-1, (C // BLOCK, BLOCK))
    e = (v.abs().amax(-1).view(torch.int32) >> 23) & 255       # biased exponent of the largest
    b = torch.where(e == 255, e, (e - 2).clamp(min=0))
    inv = ((254 - b).clamp(min=1) << 23).view(torch.float32)   # 2^(127 - b)
    v = v * inv[..., None]
    a = v.abs()
    # steps 0, .5, 1, 1.5, 2, 3, 4, 6: the borders between them, ties to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5.0)) + 8 * (v < 0).to(torch.uint8)
    code = torch.where((b == 255)[..., None], torch.zeros_like(code), code).flatten(-2)
    pad = -(C // BLOCK) % (GROUP // BLOCK)
    b = torch.nn.functional.pad(b.to(torch.uint8), (0, pad)).unflatten(-1, (-1, GROUP // BLOCK))
    return code[..., 0::2] | (code[..., 1::2] << 4), b.transpose(-3, -2).contiguous()


def _plain_values(codes, scale):
    """What MX4 codes and scales stand for, in float32."""
    steps = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    steps = torch.cat([steps, -steps])
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    b = scale.transpose(-3, -2).flatten(-2)[..., :c.shape[-1] // BLOCK].to(torch.int32)
    # 2^(b - 127); 2^-127 is below float32's normal numbers
    s = torch.where(b == 0, torch.full_like(b, 1 << 22), b << 23)
    s = torch.where(b == 255, torch.full_like(b, 0x7FC00000), s).view(torch.float32)
    return (steps[c.int()].unflatten(-1, (-1, BLOCK)) * s[..., None]).flatten(-2)


def _plain_grouped(rows, v, w):
    """rows[r] times the matrix of its expert: experts padded to the fullest."""
    c = v["case"]
    o = v["offsets"].long()
    r = torch.arange(rows.shape[0], device=DEV)
    e = torch.searchsorted(o[1:], r, right=True)
    at = r - o[e]
    slot = e if v["expert_map"] is None else v["expert_map"].long()[e]
    padded = torch.zeros((c["E"] - c["dead"], v["cap"], rows.shape[1]), device=DEV)
    padded[slot, at] = rows
    return torch.bmm(padded, w.transpose(1, 2).contiguous())[slot, at]


def _run_plain(v):
    c = v["case"]
    if c["kind"] == "quant":
        return _plain_values(*_plain_quantize(v["src"])).to(v["src"].dtype)
    token = v["row_src"].long() // c["k"]
    if c["kind"] == "product":
        x = _plain_values(*v["x"]) if c["act"] == 4 else v["x"].float()
        return _plain_grouped(x[token], v, _plain_values(*v["w"])).to(DTYPES[c["dtype"]])
    x = v["x"].float()
    if c["act"] == 4:
        x = _plain_values(*_plain_quantize(x))
    a = _plain_grouped(x[token], v, _plain_values(*v["w_gate_up"]))
    g, u = a[:, :c["f"]], a[:, c["f"]:]
    h = g / (1.0 + torch.exp(-g)) * u
    h = _plain_values(*_plain_quantize(h)) if c["act"] == 4 else h.to(torch.bfloat16).float()
    return _plain_grouped(h, v, _plain_values(*v["w_down"])).to(torch.bfloat16)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def _mx4_bytes(n):
    return n // 2 + n // BLOCK


def work(case):
    if case["kind"] == "quant":       # values in, codes and scales out and in, values out
        n = case["n"] * case["R"] * case["C"]
        return dict(bytes=2 * n * (2 if case["dtype"] == "bf16" else 4) + 2 * _mx4_bytes(n),
                    flops=8 * n)
    T, k = case["T"], case["k"]
    R = T * k
    live = min(case["E"] - case["dead"], R)       # experts with rows, at most
    if case["kind"] == "product":
        N, K = case["N"], case["K"]
        x = _mx4_bytes(T * K) if case["act"] == 4 else 2 * T * K
        es = 2 if case["dtype"] == "bf16" else 4
        return dict(bytes=x + live * _mx4_bytes(N * K) + R * N * es + 4 * R, flops=2 * R * N * K)
    d, f = case["d"], case["f"]
    return dict(bytes=2 * T * d + live * _mx4_bytes(3 * d * f) + 2 * R * d + 4 * R,
                flops=6 * R * d * f)


# ---------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------
def _exact_round(x):
    """The nearest MX4 values: per 32 columns the scale is 2^(floor(log2 amax) - 2); steps of
    1/2 up to 2, 1 up to 4, 2 up to 6."""
    v = x.double().unflatten(-1, (-1, BLOCK))
    _, e = torch.frexp(v.abs().amax(-1, keepdim=True))          # amax = m 2^e, m in [1/2, 1)
    s = ((e.long() - 3).clamp(min=-127) + 1023 << 52).view(torch.float64)
    q = v / s
    _, e = torch.frexp(q)
    step = ((e.long() - 2).clamp(min=-1) + 1023 << 52).view(torch.float64)
    return (((q / step).round() * step).clamp(-6, 6) * s).flatten(-2)


def _exact_values(codes, scale):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    m, e = (c & 1).double(), (c >> 1) & 3
    v = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2((e - 1).double()))
    v = torch.where(c >= 8, -v, v)
    G, R, _ = scale.shape[-3:]
    b = scale.movedim(-2, -3).reshape(scale.shape[:-3] + (R, G * 8))[..., :v.shape[-1] // BLOCK]
    # ldexp by exponent bits: exp2 on the device is not exact
    s = (b.long() - 127 + 1023 << 52).view(torch.float64)
    return v * s.repeat_interleave(BLOCK, dim=-1)


def exact(case, seed):
    v = _inputs(case, seed)
    if case["kind"] == "quant":
        return _exact_round(v["src"])
    o = v["offsets"].tolist()
    slots = range(case["E"]) if v["expert_map"] is None else v["expert_map"].tolist()
    token = torch.div(v["row_src"].long(), case["k"], rounding_mode="floor")

    def weights(name, e):
        return _exact_values(v[name][0][slots[e]], v[name][1][slots[e]])

    R = token.numel()
    live = [e for e in range(case["E"]) if o[e + 1] > o[e]]
    if case["kind"] == "product":
        x = _exact_values(*v["x"]) if case["act"] == 4 else v["x"].double()
        y = torch.empty((R, case["N"]), dtype=torch.float64, device=DEV)
        for e in live:
            y[o[e]:o[e + 1]] = x[token[o[e]:o[e + 1]]] @ weights("w", e).T
        return y
    x = v["x"].double()
    if case["act"] == 4:
        x = _exact_round(x)
    y = torch.empty((R, case["d"]), dtype=torch.float64, device=DEV)
    for e in live:
        a = x[token[o[e]:o[e + 1]]] @ weights("w_gate_up", e).T
        h = a[:, :case["f"]] * torch.sigmoid(a[:, :case["f"]]) * a[:, case["f"]:]
        h = _exact_round(h) if case["act"] == 4 else h.to(torch.bfloat16).double()
        y[o[e]:o[e + 1]] = h @ weights("w_down", e).T
    return y
