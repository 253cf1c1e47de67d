"""What a training step of a pre-norm MoE block does around the expert FFN, as
measurable cases: each is one pass through an operator on inputs that are
already on the GPU.

  norm          moe_layer_norm: residual add, layer norm, row statistics
  norm_bwd      moe_layer_norm_bwd: dx onto the residual's gradient, dgamma, dbeta
  balance       moe_balance_loss: loss, per-sequence expert counts, mean probabilities
  balance_train the same, then moe_balance_loss_bwd: the gradient of the logits
  act8_save     moe_act8_save and moe_act8_load: pre-activations kept in 8 bits
                with one power-of-two scale per 32, and what they stand for
  act8_bwd      moe_swiglu_bwd_act8: the SwiGLU backward at the 8-bit checkpoint

Sizes are the repository's layers (d_model 1024, 2048 and 4096, d_ff 1024 and
2048, 64 experts top-8 and top-2, 45 of 64 after pruning, 8192 tokens, shards of
32768 rows), decode batches of them, and long batches of many experts.  Values:
a residual stream with a few large channels, router logits with a skewed bias,
pre-activations of x ~ N(0, 1) through weights ~ N(0, 0.02).

With ``own`` false the operators are computed from their formulas by elementary
torch operations in float32, each output rounded once.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
COEF = 0.01
BLOCK = 32          # columns that share a scale of the 8-bit checkpoint


def listed():
    return [
        # a handful of sequences decoding, one token each: latency
        dict(name="norm_decode_8", kind="norm", T=8, d=2048, dtype="bf16", residual=True,
             beta=True),
        # an expert-parallel rank's 32768 tokens of the wide layer
        dict(name="norm_shard", kind="norm", T=32768, d=4096, dtype="bf16", residual=True,
             beta=True),
        # one prompt of odd length, fp32, a width that is no multiple of 64
        dict(name="norm_bwd_1531_f32", kind="norm_bwd", T=1531, d=1000, dtype="f32",
             dres=False, beta=True),
        # the `balanced` training step's block: 8192 tokens, d 2048
        dict(name="norm_bwd_balanced", kind="norm_bwd", T=8192, d=2048, dtype="bf16", dres=True,
             beta=True),
        # the load statistics of a decode batch
        dict(name="balance_decode_8", kind="balance", T=8, E=64, k=8, seqs=1, dead=0),
        # the `balanced` training step, loss over the whole batch
        dict(name="balance_train_8192", kind="balance_train", T=8192, E=64, k=8, seqs=1, dead=0),
        # the layer after pruning (45 experts), packed sequences of uneven length, some empty
        dict(name="balance_train_packed", kind="balance_train", T=32768, E=45, k=8, seqs=24,
             dead=0),
        # a long batch over many experts, a quarter of them pruned by mask
        dict(name="balance_train_131072", kind="balance_train", T=131072, E=256, k=8, seqs=32,
             dead=64),
        # the routed rows of a short batch of odd length, d_ff 2048
        dict(name="act8_save_1531", kind="act8_save", R=1531, f=2048, dtype="bf16"),
        # the `balanced` training step: 8192 tokens x 8 slots, d_ff 1024
        dict(name="act8_save_balanced", kind="act8_save", R=65536, f=1024, dtype="bf16"),
        # the small micro-batch's backward: 1531 tokens, top-2
        dict(name="act8_bwd_3062", kind="act8_bwd", R=3062, f=2048, dtype="bf16"),
        # the `balanced` training step's backward
        dict(name="act8_bwd_balanced", kind="act8_bwd", R=65536, f=1024, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))
    return n - 1 if n == 3072 else n    # no layer of this repository has that size


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "balance", "balance_train",
                       "balance_train", "act8_save", "act8_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = 2 if dtype == "bf16" else 4
    most = 32768 * 4096 * 2             # elements' bytes of the largest listed tensor
    if kind in ("norm", "norm_bwd"):
        d = 8 * rng.choice([rng.randint(8, 512), 16 * rng.randint(1, 32)])
        d += 8 * (d == 3072)
        c = dict(kind=kind, T=_log(rng, 1, min(65536, most // (d * es))), d=d, dtype=dtype,
                 beta=rng.random() < 0.7)
        c["residual" if kind == "norm" else "dres"] = rng.random() < 0.6
        return c
    if kind in ("balance", "balance_train"):
        E = rng.choice([8, 16, 45, 64, 128, 256, rng.randint(2, 256)])
        k = rng.choice([k for k in (1, 2, 4, 8) if k <= E // 2] or [1])
        T = _log(rng, 1, 131072)
        return dict(kind=kind, T=T, E=E, k=k, seqs=rng.choice([1, 1, rng.randint(2, 64)]),
                    dead=rng.choice([0, 0, E // 4]))
    # the largest: 65536 rows of 2048 bf16 pre-activations
    f = 32 * rng.choice([rng.randint(4, 64), 2 * rng.randint(4, 32)])
    f += 32 * (f == 1536)
    return dict(kind=kind, R=_log(rng, 1, 65536 * 2048 // (f * es)), f=f, dtype=dtype)


# ---------------------------------------------------------------------------------------
# inputs, from the seed alone
# ---------------------------------------------------------------------------------------
def _normal(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g)


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]
    v = {}
    if kind in ("norm", "norm_bwd"):
        dt, T, d = DTYPES[case["dtype"]], case["T"], case["d"]
        # a residual stream: some channels carry much larger values, rows have a mean
        scale = torch.exp(_normal(g, d, std=0.5))
        scale[torch.randint(0, d, (max(1, d // 256),), device=DEV, generator=g)] *= 20.0
        x = _normal(g, T, d) * scale + _normal(g, T, 1, std=0.2)
        v["gamma"] = 1.0 + _normal(g, d, std=0.1)
        v["beta"] = _normal(g, d, std=0.1) if case["beta"] else None
        v["x"] = x.to(dt)
        if kind == "norm":
            v["residual"] = _normal(g, T, d, std=0.5).to(dt) if case["residual"] else None
        else:
            # the statistics the forward pass left
            xf = v["x"].float()
            v["mean"] = xf.mean(1)
            v["rstd"] = torch.rsqrt(((xf - v["mean"][:, None]) ** 2).mean(1) + EPS)
            v["dy"] = _normal(g, T, d).to(dt)
            v["dres"] = _normal(g, T, d).to(dt) if case["dres"] else None
    elif kind in ("balance", "balance_train"):
        T, E, k, S = case["T"], case["E"], case["k"], case["seqs"]
        logits = _normal(g, T, E, std=0.9) + _normal(g, E, std=0.5)
        alive = None
        if case["dead"]:
            alive = torch.ones(E, dtype=torch.uint8, device=DEV)
            alive[torch.randperm(E, device=DEV, generator=g)[:case["dead"]]] = 0
            logits = logits.masked_fill(alive == 0, -math.inf)   # as the router writes them
        v["logits"], v["alive"] = logits, alive
        v["topk_idx"] = torch.topk(logits, k, dim=1).indices.to(torch.int32).contiguous()
        v["seq_offsets"] = None
        if S > 1:
            # cut points anywhere: lengths from none to many
            cut = torch.randint(0, T + 1, (S - 1,), device=DEV, generator=g).sort().values
            v["seq_offsets"] = torch.cat([cut.new_zeros(1), cut, cut.new_full((1,), T)]).to(
                torch.int32)
        v["dloss"] = torch.full((1,), 0.5, device=DEV)
    else:
        dt, R, f = DTYPES[case["dtype"]], case["R"], case["f"]
        act = _normal(g, R, 2 * f, std=0.9).to(dt)
        if kind == "act8_save":
            v["act"] = act
        else:
            v["q"], v["scale"] = _plain_save(act)
            v["dh"] = _normal(g, R, f, std=0.05).to(dt)
    return v


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    if own:
        state["out"] = _buffers(case, state)
    return state


def _buffers(case, v):
    """The output buffers and workspaces that a program keeps from call to call."""
    import paper_2601_14327_amd as laep

    kind = case["kind"]
    f32 = torch.float32
    if kind == "norm":
        b = dict(out=torch.empty_like(v["x"]),
                 mean=torch.empty(case["T"], dtype=f32, device=DEV),
                 rstd=torch.empty(case["T"], dtype=f32, device=DEV))
        if v["residual"] is not None:
            b["sum_out"] = torch.empty_like(v["x"])
        return b
    if kind == "norm_bwd":
        n = laep.workspace_bytes(laep.LAEP_CALL_LAYER_NORM_BWD, case["T"], 1, 1, case["d"])
        return dict(dx=torch.empty_like(v["x"]), dgamma=torch.empty_like(v["gamma"]),
                    dbeta=torch.empty_like(v["gamma"]) if case["beta"] else None,
                    ws=torch.empty(max(n, 1), dtype=torch.uint8, device=DEV))
    if kind in ("balance", "balance_train"):
        S, E = case["seqs"], case["E"]
        n = laep.workspace_bytes(laep.LAEP_CALL_BALANCE, case["T"], S, E)
        b = dict(loss=torch.empty(1, dtype=f32, device=DEV),
                 counts=torch.empty((S, E), dtype=torch.int32, device=DEV),
                 prob_mean=torch.empty((S, E), dtype=f32, device=DEV),
                 grad_coef=torch.empty((S, E), dtype=f32, device=DEV),
                 ws=torch.empty(max(n, 1), dtype=torch.uint8, device=DEV))
        if kind == "balance_train":
            return b, torch.empty_like(v["logits"])
        return b, None
    dt, R, f = DTYPES[case["dtype"]], case["R"], case["f"]
    if kind == "act8_save":
        return dict(q=torch.empty((R, 2 * f), dtype=torch.int8, device=DEV),
                    scale=torch.empty((R, 2 * f // BLOCK), dtype=torch.uint8, device=DEV),
                    act=torch.empty((R, 2 * f), dtype=dt, device=DEV))
    return dict(da=torch.empty((R, 2 * f), dtype=dt, device=DEV),
                h=torch.empty((R, f), dtype=dt, device=DEV))


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(v):
    import paper_2601_14327_amd as laep

    kind, b = v["case"]["kind"], v["out"]
    if kind == "norm":
        return laep.moe_layer_norm(v["x"], v["gamma"], v["beta"], residual=v["residual"], eps=EPS,
                                   **b)
    if kind == "norm_bwd":
        return laep.moe_layer_norm_bwd(v["dy"], v["x"], v["gamma"], v["mean"], v["rstd"],
                                       dres=v["dres"], want_dbeta=v["beta"] is not None, **b)
    if kind in ("balance", "balance_train"):
        fwd, dlogits = b
        loss, counts, prob, coef = laep.moe_balance_loss(
            v["logits"], v["topk_idx"], coef=COEF, alive=v["alive"],
            seq_offsets=v["seq_offsets"], **fwd)
        if kind == "balance":
            return loss, counts, prob
        dl = laep.moe_balance_loss_bwd(v["logits"], coef, dloss=v["dloss"], alive=v["alive"],
                                       seq_offsets=v["seq_offsets"], dlogits=dlogits)
        return loss, counts, prob, dl
    if kind == "act8_save":
        q, scale = laep.moe_act8_save(v["act"], q=b["q"], scale=b["scale"])
        return laep.moe_act8_load(q, scale, v["act"].dtype, out=b["act"])
    return laep.moe_swiglu_bwd_act8(v["q"], v["scale"], v["dh"], **b)


def _plain_save(act):
    R, C = act.shape
    x = act.float().reshape(R, C // BLOCK, BLOCK)
    amax = x.abs().amax(2)
    e = (amax.view(torch.int32) >> 23) & 255          # biased exponent of the largest
    b = torch.where(e == 255, e, (e - 6).clamp(min=1))
    inv = ((254 - b).clamp(min=1) << 23).view(torch.float32)      # 2^(127 - b)
    q = torch.round(x * inv[..., None]).clamp(-127, 127)
    q = torch.where((b == 255)[..., None], torch.zeros_like(q), q)
    return q.to(torch.int8).reshape(R, C), b.to(torch.uint8)


def _plain_load(q, scale):
    R, C = q.shape
    b = scale.to(torch.int32)
    s = torch.where(b == 255, torch.full_like(b, 0x7FC00000), b << 23).view(torch.float32)
    return (q.float().reshape(R, C // BLOCK, BLOCK) * s[..., None]).reshape(R, C)


def _plain_probs(logits, alive):
    if alive is not None:
        logits = logits.masked_fill(alive == 0, -math.inf)
    m = logits.amax(1, keepdim=True)
    p = torch.exp(logits - torch.where(m == -math.inf, torch.zeros_like(m), m))
    z = p.sum(1, keepdim=True)
    return p / torch.where(z == 0, torch.ones_like(z), z)


def _sequence_of(v):
    """The sequence of each token, and the sequences' lengths."""
    T, S = v["case"]["T"], v["case"]["seqs"]
    if S == 1:
        return (torch.zeros(T, dtype=torch.int64, device=DEV),
                torch.full((1,), T, dtype=torch.int64, device=DEV))
    o = v["seq_offsets"].long()
    seq = torch.searchsorted(o[1:], torch.arange(T, device=DEV), right=True)
    return seq, o[1:] - o[:-1]


def _run_plain(v):
    c = v["case"]
    kind = c["kind"]
    if kind == "norm":
        x = v["x"]
        s = x if v["residual"] is None else (x.float() + v["residual"].float()).to(x.dtype)
        sf = s.float()
        mean = sf.mean(1)
        cen = sf - mean[:, None]
        rstd = 1.0 / torch.sqrt((cen * cen).mean(1) + EPS)
        y = cen * rstd[:, None] * v["gamma"]
        if v["beta"] is not None:
            y = y + v["beta"]
        return y.to(x.dtype), s, mean, rstd
    if kind == "norm_bwd":
        x, dy = v["x"].float(), v["dy"].float()
        xh = (x - v["mean"][:, None]) * v["rstd"][:, None]
        g = dy * v["gamma"]
        dx = v["rstd"][:, None] * (g - g.mean(1, keepdim=True)
                                   - xh * (g * xh).mean(1, keepdim=True))
        if v["dres"] is not None:
            dx = dx + v["dres"].float()
        return (dx.to(v["x"].dtype), (dy * xh).sum(0),
                dy.sum(0) if v["beta"] is not None else None)
    if kind in ("balance", "balance_train"):
        T, E, k, S = c["T"], c["E"], c["k"], c["seqs"]
        seq, n = _sequence_of(v)
        p = _plain_probs(v["logits"], v["alive"])
        nf = n.clamp(min=1).float()[:, None]
        prob = torch.zeros((S, E), device=DEV).index_add_(0, seq, p) / nf
        cell = (seq[:, None] * E + v["topk_idx"].long()).reshape(-1)
        counts = torch.zeros(S * E, dtype=torch.int32, device=DEV).index_add_(
            0, cell, torch.ones_like(cell, dtype=torch.int32)).reshape(S, E)
        n_alive = E if v["alive"] is None else (v["alive"] != 0).sum().float()
        live = (n > 0).sum().float()
        frac = counts.float() * n_alive / (k * nf)
        loss = COEF * (frac * prob).sum().reshape(1) / live
        if kind == "balance":
            return loss, counts, prob
        coef = (COEF * frac / (nf * live))[seq]
        dl = v["dloss"] * p * (coef - (p * coef).sum(1, keepdim=True))
        return loss, counts, prob, dl
    if kind == "act8_save":
        q, scale = _plain_save(v["act"])
        return _plain_load(q, scale).to(v["act"].dtype)
    dh = v["dh"].float()
    f = dh.shape[1]
    a = _plain_load(v["q"], v["scale"])
    ag, au = a[:, :f], a[:, f:]
    sg = 1.0 / (1.0 + torch.exp(-ag))
    sl = ag * sg
    da = torch.cat([dh * au * sg * (1.0 + ag * (1.0 - sg)), dh * sl], 1)
    return da.to(v["dh"].dtype), (sl * au).to(v["dh"].dtype)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_bwd"):
        T, d = case["T"], case["d"]
        n = T * d * (2 if case["dtype"] == "bf16" else 4)
        params = 4 * d * (2 if case["beta"] else 1)
        if kind == "norm":      # x (and the residual) in, y (and the sum) out, statistics
            return dict(bytes=n * (4 if case["residual"] else 2) + 8 * T + params,
                        flops=8 * T * d)
        return dict(bytes=n * (4 if case["dres"] else 3) + 8 * T + 4 * d + params,
                    flops=14 * T * d)
    if kind in ("balance", "balance_train"):
        T, E, k, S = case["T"], case["E"], case["k"], case["seqs"]
        b = 4 * T * E + 4 * T * k + 8 * S * E
        if kind == "balance":
            return dict(bytes=b, flops=5 * T * E)
        return dict(bytes=b + 4 * T * E, flops=12 * T * E)
    R, f = case["R"], case["f"]
    es = 2 if case["dtype"] == "bf16" else 4
    ckpt = R * 2 * f + R * 2 * f // BLOCK
    if kind == "act8_save":     # values in, the checkpoint written and read, values out
        return dict(bytes=2 * R * 2 * f * es + 2 * ckpt, flops=4 * R * 2 * f)
    return dict(bytes=ckpt + 4 * R * f * es, flops=16 * R * f)


# ---------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------
def exact(case, seed):
    v = _inputs(case, seed)
    kind = case["kind"]
    if kind == "norm":
        s = v["x"].double()
        if v["residual"] is not None:
            s = (s + v["residual"].double()).to(v["x"].dtype).double()   # the sum is stored
        var, mean = torch.var_mean(s, dim=1, correction=0)
        rstd = (var + EPS) ** -0.5
        y = (s - mean.unsqueeze(1)) * rstd.unsqueeze(1) * v["gamma"].double()
        return (y if v["beta"] is None else y + v["beta"].double()), s, mean, rstd
    if kind == "norm_bwd":
        # dx = rstd (I - 11'/d - xh xh'/d) (gamma * dy)
        d = case["d"]
        dy = v["dy"].double()
        rstd = v["rstd"].double().unsqueeze(1)
        xh = (v["x"].double() - v["mean"].double().unsqueeze(1)) * rstd
        w = dy * v["gamma"].double()
        along = (w * xh).sum(1, keepdim=True) / d
        dx = rstd * (w - w.sum(1, keepdim=True) / d - along * xh)
        if v["dres"] is not None:
            dx += v["dres"].double()
        return dx, (xh * dy).sum(0), dy.sum(0) if case["beta"] else None
    if kind in ("balance", "balance_train"):
        T, E, k, S = case["T"], case["E"], case["k"], case["seqs"]
        l = v["logits"].double()
        alive = torch.ones(E, dtype=torch.bool, device=DEV)
        if v["alive"] is not None:
            alive = v["alive"].bool()
        p = torch.zeros_like(l)
        p[:, alive] = torch.softmax(l[:, alive], dim=1)
        bounds = [0, T] if S == 1 else v["seq_offsets"].tolist()
        counts = torch.zeros((S, E), dtype=torch.int32, device=DEV)
        prob = torch.zeros((S, E), dtype=torch.float64, device=DEV)
        dl = torch.zeros_like(l)
        live = sum(b > a for a, b in zip(bounds, bounds[1:]))
        loss = torch.zeros(1, dtype=torch.float64, device=DEV)
        for s, (a, b) in enumerate(zip(bounds, bounds[1:])):
            if a == b:
                continue
            counts[s] = torch.bincount(v["topk_idx"][a:b].reshape(-1), minlength=E).to(torch.int32)
            prob[s] = p[a:b].mean(0)
            f = counts[s].double() * (int(alive.sum()) / (k * (b - a)))
            loss += COEF * (f @ prob[s]) / live
            w = f * (COEF / (live * (b - a)))
            dl[a:b] = p[a:b] * (w - (p[a:b] * w).sum(1, keepdim=True))
        if kind == "balance":
            return loss, counts, prob
        return loss, counts, prob, dl * v["dloss"].double()
    if kind == "act8_save":
        x = v["act"].double().unflatten(1, (-1, BLOCK))
        top = x.abs().amax(2, keepdim=True)
        _, e = torch.frexp(top)                       # top = m 2^e, m in [1/2, 1)
        # 2^(e - 7) from its bits: the device's pow is not exact, and bf16 values tie often
        step = ((e.long() - 7).clamp(min=-126) + 1023 << 52).view(torch.float64)
        return ((x / step).round().clamp(-127, 127) * step).flatten(1)
    a = v["q"].double().unflatten(1, (-1, BLOCK))
    a = (a * torch.exp2(v["scale"].double() - 127.0).unsqueeze(2)).flatten(1)
    g, u = a.chunk(2, dim=1)
    dh = v["dh"].double()
    sg = torch.sigmoid(g)
    return torch.cat([dh * u * (sg + g * sg * (1.0 - sg)), dh * g * sg], 1), g * sg * u
