"""Operators of a training pass beside those of operators.py, as measured: what they compute in plain torch, the calls a
user makes of the framework, and the sizes that stand for their use.

  norm         RMS or layer norm of rows, with the residual addition before it and the statistics that the gradient needs
  norm_grad    its gradient: dx (with the residual's gradient added) and the weight's, summed over the rows
  norm_step    both
  rope         rotation of the heads of q and k by their positions, or back (the gradient); half and interleaved layouts,
               part of the head, frequencies scaled for long contexts
  router       softmax over the experts, the k largest, their weights, counts, offsets, balance loss and z loss
  router_grad  the gradient of the logits through the weights and both losses
  router_step  both
  policy       clipped policy loss with a KL term towards a reference, and its gradient to the log-probs

Shapes are those of workloads.py: hidden 2048, 32 query and 4 key heads of 128, 128 experts with 8 for each token, chunks of
2048 tokens, 64 sequences, responses in segments of up to 16384 tokens, groups of 8; and odd sizes beside them.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = dict(bf16=torch.bfloat16, fp16=torch.float16, fp32=torch.float32)


def listed():
    return [
        # a small model's layer norm in fp32, forward and backward: odd sizes, latency
        dict(name="norm_step small", kind="norm_step", norm="layer", rows=203, heads=1, width=1111, pad=0, x="fp32", y="fp32",
             w="fp32", add=False, bias=True),
        # a training micro-batch of 16 chunks: residual addition and norm, bf16
        dict(name="norm batch", kind="norm", norm="rms", rows=32768, heads=1, width=2048, pad=0, x="bf16", y="bf16", w="bf16",
             add=True, bias=False),
        # the same rows' backward pass, with the gradient of the residual stream coming in
        dict(name="norm_grad batch", kind="norm_grad", norm="rms", rows=32768, heads=1, width=2048, pad=0, x="bf16", y="bf16",
             w="bf16", add=True, bias=False),
        # the per-head norm of 32 query heads inside the projection's rows of 5120: many short rows, one small weight
        dict(name="norm_grad heads", kind="norm_grad", norm="rms", rows=16384, heads=32, width=128, pad=1024, x="bf16", y="bf16",
             w="bf16", add=False, bias=False),
        # one chunk of 2048 tokens on the way forward
        dict(name="rope chunk", kind="rope", rows=2048, q=32, k=4, dim=128, rotary=128, layout="half", scaling="none", factor=1.0,
             farthest=32768, type="bf16", inverse=False),
        # far positions of a stretched context, interleaved pairs, part of the head, fp32, back
        dict(name="rope far", kind="rope", rows=777, q=9, k=0, dim=96, rotary=64, layout="interleaved", scaling="parts", factor=8.0,
             farthest=1_000_000, type="fp32", inverse=True),
        # the gradients of a packed micro-batch of 65536 tokens
        dict(name="rope batch", kind="rope", rows=65536, q=32, k=4, dim=128, rotary=128, layout="half", scaling="none", factor=1.0,
             farthest=65536, type="bf16", inverse=True),
        # 64 tokens, one of each live sequence: latency, forward and backward
        dict(name="router_step small", kind="router_step", rows=64, experts=128, k=8, type="fp32", padded=0.0, renormalise=True,
             z=0.0),
        # a packed micro-batch of 131072 tokens
        dict(name="router batch", kind="router", rows=131072, experts=128, k=8, type="fp32", padded=0.1, renormalise=True, z=1e-3),
        # its gradient, logits in bf16 (equal logits are common there)
        dict(name="router_grad batch", kind="router_grad", rows=131072, experts=128, k=8, type="bf16", padded=0.0, renormalise=True,
             z=1e-3),
        # one group of 8 short responses
        dict(name="policy group", kind="policy", seqs=8, rows=2100, masked=0.3, reduce="sequences", per_token=False, kl=0.0, ref=False),
        # 128 prompts x 8 responses of a segment, a third prompt tokens
        dict(name="policy batch", kind="policy", seqs=1024, rows=4_000_000, masked=0.33, reduce="tokens", per_token=False, kl=1e-3,
             ref=True),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "rope", "router", "policy"])
    if kind in ("norm", "router"):
        kind += rng.choice(["", "_grad", "_step"])
    if kind.startswith("norm"):
        heads = rng.choice([1, 1, rng.randint(2, 40)])
        width = rng.choice([8 * size(8, 512), 8 * size(8, 1024), size(1, 4099)]) if heads == 1 else rng.choice([64, 96, 128, 256])
        x, y = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32"), ("fp16", "fp16")])
        norm = rng.choice(["rms", "rms", "layer"])
        return dict(kind=kind, norm=norm, rows=size(1, max(1, min(32768, 30_000_000 // (heads * width)))), heads=heads, width=width,
                    pad=rng.choice([0, 0, 8 * rng.randint(1, 64)]), x=x, y=y, w=rng.choice(["bf16", "fp32"]),
                    add=heads == 1 and rng.random() < 0.5, bias=norm == "layer" and rng.random() < 0.7)
    if kind == "rope":
        dim = rng.choice([64, 128, 128, 80, 96, 256])
        q, k = rng.choice([(32, 4), (16, 2), (4, 1), (rng.randint(1, 40), rng.randint(0, 8))])
        t = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        return dict(kind=kind, rows=size(1, min(65536, 150_000_000 // ((q + k) * dim))), q=q, k=k, dim=dim,
                    rotary=rng.choice([dim, dim, dim // 2]), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "base", "parts"]), factor=rng.choice([2.0, 4.0, 8.0]),
                    farthest=size(100, 1_000_000), type=t, inverse=rng.random() < 0.5)
    if kind.startswith("router"):
        experts = rng.choice([8, 16, 60, 64, 128, 128, 256, 384, rng.randint(2, 512)])
        return dict(kind=kind, rows=size(1, min(131072, 16_000_000 // experts)), experts=experts,
                    k=min(experts, rng.choice([1, 2, 4, 6, 8, 8, 10])), type=rng.choice(["fp32", "fp32", "bf16", "fp16"]),
                    padded=round(rng.choice([0.0, rng.uniform(0, 0.5)]), 2), renormalise=rng.random() < 0.7,
                    z=rng.choice([0.0, 1e-3]))
    seqs = size(1, 1024)
    return dict(kind=kind, seqs=seqs, rows=size(seqs, 4_000_000), masked=round(rng.uniform(0, 0.6), 2),
                reduce=rng.choice(["tokens", "sequences", "sum"]), per_token=rng.random() < 0.3, kl=rng.choice([0.0, 1e-3, 0.04]),
                ref=rng.random() < 0.6)


# ----------------------------------------------------------------------------------------------- inputs

EPS = 1e-6
THETA = 1e6
TRAINED = 32768                  # positions that the frequencies were trained on, where they are stretched
FAST, SLOW = 32.0, 1.0           # turns over those positions from which on / up to which a pair is kept / stretched in full
CLIP_LOW, CLIP_HIGH = 0.2, 0.28
BALANCE = 1e-2


def _seeded(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, *shape, std=1.0, mean=0.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV).mul_(std).add_(mean).to(dtype)


def _rows_of(buffer, case):
    """[rows, width], or [rows, heads, width], inside the wider rows of a buffer."""
    n = case["heads"] * case["width"]
    t = buffer[:, :n]
    return t if case["heads"] == 1 else t.unflatten(1, (case["heads"], case["width"]))


def _prepare_norm(case, seed):
    g = _seeded(seed)
    wide = (case["rows"], case["heads"] * case["width"] + case["pad"])
    xt, yt, wt = TYPES[case["x"]], TYPES[case["y"]], TYPES[case["w"]]
    s = dict(x=_rows_of(_normal(g, *wide, std=1.5, mean=0.2, dtype=xt), case),
             weight=_normal(g, case["width"], std=0.1, mean=1.0, dtype=wt),
             bias=_normal(g, case["width"], std=0.1, dtype=wt) if case["bias"] else None)
    if case["kind"] != "norm_grad" and case["add"]:
        s["add"] = _rows_of(_normal(g, *wide, std=0.5, dtype=yt), case)
    if case["kind"] != "norm":
        s["dy"] = _rows_of(_normal(g, *wide, std=1e-2, dtype=yt), case)
        if case["add"]:
            s["d_sum"] = _rows_of(_normal(g, *wide, std=1e-2, dtype=xt), case)
    if case["kind"] == "norm_grad":                       # the statistics that the forward pass kept
        mean, rstd = _statistics(s["x"], case["norm"])
        s.update(mean=mean, rstd=rstd)
    return s


def _statistics(x, norm):
    f = x.float()
    mean = f.mean(dim=-1) if norm == "layer" else None
    var = (f if mean is None else f - mean[..., None]).square().mean(dim=-1)
    return mean, torch.rsqrt(var + EPS)


def _prepare_rope(case, seed):
    g = _seeded(seed)
    n, t = case["rows"], TYPES[case["type"]]
    qkv = _normal(g, n, (case["q"] + 2 * case["k"]) * case["dim"], dtype=t)           # q, k and v rows of one projection
    q, k, _ = qkv.split([case["q"] * case["dim"], case["k"] * case["dim"], case["k"] * case["dim"]], dim=1)
    # packed responses: runs of consecutive positions, each from a place of its own
    run = max(1, n // 7)
    first = torch.randint(max(1, case["farthest"] - run), (-(-n // run),), generator=g, device=DEV)
    at = torch.arange(n, device=DEV)
    s = dict(q=q.unflatten(1, (case["q"], case["dim"])), positions=(first[at // run] + at % run).to(torch.int32))
    s["k"] = k.unflatten(1, (case["k"], case["dim"])) if case["k"] else None
    s["frequencies"] = _frequencies(case)
    return s


def _frequencies(case):
    """Angle of every pair for one position, in 64 bits."""
    d, factor = case["rotary"], case["factor"]
    i = torch.arange(0, d, 2, dtype=torch.float64, device=DEV)
    if case["scaling"] == "base":
        return (THETA * factor ** (d / (d - 2))) ** (-i / d) if d > 2 else THETA ** (-i / d)
    f = THETA ** (-i / d)
    if case["scaling"] == "linear":
        return f / factor
    if case["scaling"] == "parts":
        turns = TRAINED * f / (2 * math.pi)
        keep = ((turns - SLOW) / (FAST - SLOW)).clamp(0, 1)
        return f * (keep + (1 - keep) / factor)
    return f


def _scale(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "parts" else 1.0


def _prepare_router(case, seed):
    g = _seeded(seed)
    T, E = case["rows"], case["experts"]
    logits = (_normal(g, T, E, std=1.2) + _normal(g, E, std=0.4)).to(TYPES[case["type"]])
    live = None
    if case["padded"] > 0:
        live = torch.rand(T, generator=g, device=DEV) >= case["padded"]
    s = dict(logits=logits, live=live)
    if case["kind"] != "router":
        s["d_weights"] = _normal(g, T, case["k"], std=1e-3)
    if case["kind"] == "router_grad":                     # what the forward pass kept
        s.update({n: v for n, v in _route(case, s).items() if n in ("idx", "lse", "counts")})
    return s


def _lengths(case, seed):
    r = random.Random(int(seed) * 13 + 5)
    share = [math.exp(0.6 * r.gauss(0, 1)) if r.random() > 0.03 else 0.0 for _ in range(case["seqs"])]
    share[-1] += 1e-3
    total, got = sum(share), [0] * case["seqs"]
    for i, v in enumerate(share):
        got[i] = int(case["rows"] * v / total)
    got[-1] += case["rows"] - sum(got)
    return got


def _prepare_policy(case, seed):
    g = _seeded(seed)
    n = case["rows"]
    off = torch.zeros(case["seqs"] + 1, dtype=torch.int64)
    off[1:] = torch.tensor(_lengths(case, seed)).cumsum(0)
    old = -_normal(g, n).abs_() ** 3 * 0.5                # most tokens near certain, a few far from it
    lp = (old + _normal(g, n) * (0.15 * old.abs()).clamp(max=0.6)).clamp_(max=0)
    targets = torch.randint(151936, (n,), generator=g, device=DEV, dtype=torch.int32)
    targets[torch.rand(n, generator=g, device=DEV) < case["masked"]] = -1
    s = dict(lp=lp, old=old, targets=targets, off=off.to(DEV, torch.int32), most=int((off[1:] - off[:-1]).max()),
             adv=_normal(g, n if case["per_token"] else case["seqs"]))
    s["ref"] = (lp + _normal(g, n) * 0.1).clamp_(max=0) if case["ref"] else None
    s["scale"] = 1.0 if case["reduce"] != "sum" else 1.0 / max(1, n)
    return s


def prepare(case, seed):
    kind = case["kind"]
    make = _prepare_norm if "norm" in kind else _prepare_rope if kind == "rope" else _prepare_router if "router" in kind else _prepare_policy
    s = make(case, seed)
    s["case"] = case
    if own:
        s.update(_own_handle(case, s))
    return s


def _own_handle(case, s):
    """The handle and the output tensors that a program keeps beside its inputs."""
    from paper_2511_11373_b200 import binding
    kind, f32, i32 = case["kind"], dict(device=DEV), dict(dtype=torch.int32, device=DEV)
    if "norm" in kind:
        got = dict(handle=binding.Train(max_width=case["width"], device=DEV))
        rows, yt = s["x"].shape[:-1], TYPES[case["y"]]
        if kind != "norm_grad":
            got.update(y=torch.empty(s["x"].shape, dtype=yt, device=DEV), rstd=torch.empty(rows, **f32),
                       mean=torch.empty(rows, **f32) if case["norm"] == "layer" else None,
                       sum=torch.empty(s["x"].shape, dtype=s["x"].dtype, device=DEV) if case["add"] else None)
        if kind != "norm":
            got.update(dx=torch.empty(s["x"].shape, dtype=s["x"].dtype, device=DEV), dw=torch.empty(case["width"], **f32),
                       db=torch.empty(case["width"], **f32) if case["bias"] else None)
        return got
    if kind == "rope":
        handle = binding.Rope(case["rotary"], theta=THETA, layout=case["layout"], scaling=case["scaling"], factor=case["factor"],
                              trained_positions=TRAINED, fast=FAST, slow=SLOW, scale=_scale(case), device=DEV)
        return dict(handle=handle, out_q=torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEV),
                    out_k=None if s["k"] is None else torch.empty(s["k"].shape, dtype=s["k"].dtype, device=DEV))
    if "router" in kind:
        T, E, k = case["rows"], case["experts"], case["k"]
        got = dict(handle=binding.Train(max_experts=E, device=DEV))
        if kind != "router_grad":
            got.update(idx=torch.empty(T, k, **i32), weights=torch.empty(T, k, **f32), lse=torch.empty(T, **f32),
                       counts=torch.empty(E, **i32), offsets=torch.empty(E + 1, **i32), prob_sums=torch.empty(E, **f32),
                       losses=torch.empty(2, **f32))
        if kind != "router":
            got.update(d_logits=torch.empty_like(s["logits"]))
        return got
    return dict(handle=binding.Train(max_seqs=case["seqs"], device=DEV), stats=torch.empty(6, **f32),
                d_lp=torch.empty(case["rows"], **f32))


# ------------------------------------------------------------------------------------------------- run

def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    return (_plain_norm if "norm" in kind else _plain_rope if kind == "rope" else _plain_router if "router" in kind else _plain_policy)(s)


def _run_own(s):
    from paper_2511_11373_b200 import binding
    c, u, st, got = s["case"], s["handle"], 0, {}
    kind = c["kind"]
    if "norm" in kind:
        form = binding.MARS_NORM_RMS if c["norm"] == "rms" else binding.MARS_NORM_LAYER
        x = s["x"]
        if kind != "norm_grad":
            st = binding.mars_norm(u, form, x, s["weight"], EPS, s["y"], rstd=s["rstd"], mean=s["mean"], bias=s["bias"],
                                   add=s.get("add"), out_sum=s["sum"])
            got.update({n: s[n] for n in ("y", "rstd", "mean", "sum") if s[n] is not None})
            x = x if s["sum"] is None else s["sum"]
        if kind != "norm":
            st = st or binding.mars_norm_grad(u, form, s["dy"], x, s["weight"], s["rstd"], s["dx"], s["dw"], mean=s["mean"],
                                              db=s["db"], d_sum=s.get("d_sum"))
            got.update({n: s[n] for n in ("dx", "dw", "db") if s[n] is not None})
    elif kind == "rope":
        st = binding.mars_rope(u, s["positions"], s["q"], s["out_q"], s["k"], s["out_k"], inverse=c["inverse"])
        got.update({n: s[n] for n in ("out_q", "out_k") if s[n] is not None})
    elif "router" in kind:
        if kind != "router_grad":
            st = binding.mars_router(u, s["logits"], s["idx"], s["weights"], s["lse"], s["counts"], s["offsets"], s["prob_sums"],
                                     s["losses"], live=s["live"], renormalise=c["renormalise"])
            got.update({n: s[n] for n in ("idx", "weights", "lse", "counts", "offsets", "prob_sums", "losses")})
        if kind != "router":
            st = st or binding.mars_router_grad(u, s["logits"], s["idx"], s["lse"], s["counts"], s["d_logits"],
                                                d_weights=s["d_weights"], balance_coef=BALANCE, z_coef=c["z"],
                                                renormalise=c["renormalise"])
            got.update(d_logits=s["d_logits"])
    else:
        st = binding.mars_policy_loss(u, s["lp"], s["old"], s["adv"], s["targets"], s["off"], s["stats"], s["d_lp"],
                                      ref_logprobs=s["ref"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                                      kl_coef=c["kl"] if c["ref"] else 0.0,
                                      reduce=c["reduce"], scale=s["scale"], per_token=c["per_token"])
        got.update(stats=s["stats"], d_lp=s["d_lp"])
    if st:
        raise RuntimeError("status %d" % st)
    return got


def _plain_norm(s):
    c, got = s["case"], {}
    layer, x = c["norm"] == "layer", s["x"]
    if c["kind"] != "norm_grad":
        if "add" in s:
            x = (x.float() + s["add"].float()).to(x.dtype)          # the norm is that of the stored sum
            got["sum"] = x
        mean, rstd = _statistics(x, c["norm"])
        xhat = (x.float() - (mean[..., None] if layer else 0.0)) * rstd[..., None]
        y = xhat * s["weight"].float()
        if s["bias"] is not None:
            y = y + s["bias"].float()
        got.update(y=y.to(TYPES[c["y"]]), rstd=rstd)
        if layer:
            got["mean"] = mean
    else:
        mean, rstd = s["mean"], s["rstd"]
    if c["kind"] != "norm":
        xhat = (x.float() - (mean[..., None] if layer else 0.0)) * rstd[..., None]
        dy = s["dy"].float()
        g = dy * s["weight"].float()
        dx = g - xhat * (g * xhat).mean(dim=-1, keepdim=True)
        if layer:
            dx = dx - g.mean(dim=-1, keepdim=True)
        dx = dx * rstd[..., None]
        if "d_sum" in s:
            dx = dx + s["d_sum"].float()
        got.update(dx=dx.to(x.dtype), dw=(dy * xhat).reshape(-1, c["width"]).sum(dim=0))
        if c["bias"]:
            got["db"] = dy.reshape(-1, c["width"]).sum(dim=0)
    return got


def _plain_rope(s):
    c, got = s["case"], {}
    angle = s["positions"].double()[:, None] * s["frequencies"]
    sign = -1.0 if c["inverse"] else 1.0
    cos, sin = (angle.cos() * _scale(c)).float()[:, None], (angle.sin() * (sign * _scale(c))).float()[:, None]
    for name in ("q", "k"):
        t = s[name]
        if t is None:
            continue
        out, r, h = t.clone(memory_format=torch.contiguous_format), c["rotary"], c["rotary"] // 2
        a, b = (t[..., :h], t[..., h:r]) if c["layout"] == "half" else (t[..., 0:r:2], t[..., 1:r:2])
        a, b = a.float(), b.float()
        first, second = (a * cos - b * sin).to(t.dtype), (b * cos + a * sin).to(t.dtype)
        if c["layout"] == "half":
            out[..., :h], out[..., h:r] = first, second
        else:
            out[..., 0:r:2], out[..., 1:r:2] = first, second
        got["out_" + name] = out
    return got


def _route(case, s):
    z = s["logits"].float()
    T, E, k = case["rows"], case["experts"], case["k"]
    live = torch.ones(T, dtype=torch.bool, device=DEV) if s["live"] is None else s["live"]
    lse = torch.logsumexp(z, dim=1)
    p = torch.exp(z - lse[:, None])
    idx = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]          # ties: the lower index first
    w = p.gather(1, idx)
    if case["renormalise"]:
        w = w / w.sum(dim=1, keepdim=True)
    counts = torch.zeros(E, dtype=torch.int32, device=DEV)
    counts.index_add_(0, idx[live].reshape(-1), torch.ones(1, dtype=torch.int32, device=DEV).expand(int(live.sum()) * k))
    n = live.sum().clamp(min=1)
    sums = torch.where(live[:, None], p, 0.0).sum(dim=0)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = counts.cumsum(0)
    balance = E * (counts.float() / (n * k) * (sums / n)).sum()
    z_loss = torch.where(live, lse, 0.0).square().sum() / n
    return dict(idx=torch.where(live[:, None], idx, -1).to(torch.int32), weights=torch.where(live[:, None], w, 0.0),
                lse=torch.where(live, lse, 0.0), counts=counts, offsets=offsets, prob_sums=sums,
                losses=torch.stack([balance, z_loss]))


def _plain_router(s):
    c = s["case"]
    got = _route(c, s) if c["kind"] != "router_grad" else {}
    if c["kind"] == "router":
        return got
    idx, lse, counts = (got or s)["idx"], (got or s)["lse"], (got or s)["counts"]
    z, at = s["logits"].float(), idx.clamp(min=0).long()
    live, E = idx[:, 0] >= 0, c["experts"]
    total = counts.sum()
    n = (total / c["k"]).clamp(min=1)
    p = torch.exp(z - lse[:, None])
    g = BALANCE * E / n * (counts.float() / total.clamp(min=1))
    d = p * (g - (p * g).sum(dim=1, keepdim=True)) + p * (2 * c["z"] / n * lse)[:, None]
    chosen, dw = p.gather(1, at), s["d_weights"]
    if c["renormalise"]:
        w = chosen / chosen.sum(dim=1, keepdim=True)
        d.scatter_add_(1, at, w * (dw - (w * dw).sum(dim=1, keepdim=True)))
    else:
        d = d - p * (chosen * dw).sum(dim=1, keepdim=True)
        d.scatter_add_(1, at, chosen * dw)
    got["d_logits"] = torch.where(live[:, None], d, 0.0).to(s["logits"].dtype)
    return got


def _plain_policy(s):
    c = s["case"]
    n, seqs, off = c["rows"], c["seqs"], s["off"].long()
    live = s["targets"] >= 0
    seq = torch.searchsorted(off[1:].contiguous(), torch.arange(n, device=DEV), right=True)
    tokens = torch.zeros(seqs, dtype=torch.int64, device=DEV).index_add_(0, seq, live.long())
    if c["reduce"] == "tokens":
        share = (s["scale"] / live.sum().clamp(min=1)).expand(n)
    elif c["reduce"] == "sequences":
        share = (s["scale"] / (tokens > 0).sum().clamp(min=1) / tokens.clamp(min=1))[seq]
    else:
        share = torch.full((1,), s["scale"], device=DEV).expand(n)
    share = torch.where(live, share.float(), 0.0)
    adv = s["adv"] if c["per_token"] else s["adv"][seq]
    r = torch.exp(s["lp"] - s["old"])
    exact = torch.exp(s["lp"].double() - s["old"].double())          # which side of the border
    high, low = exact > 1 + CLIP_HIGH, exact < 1 - CLIP_LOW
    cut = (high & (adv > 0)) | (low & (adv < 0))
    policy = -torch.where(cut, torch.where(high, 1 + CLIP_HIGH, 1 - CLIP_LOW), r) * adv
    d = torch.where(cut, 0.0, -adv * r)
    kl = torch.zeros(n, device=DEV)
    if s["ref"] is not None:
        x = s["ref"].double() - s["lp"].double()
        kl = (torch.expm1(x) - x).float()
        d = d - c["kl"] * torch.expm1(x).float()
    every = live.sum().clamp(min=1)

    def mean(v):
        return torch.where(live, v, 0.0).double().sum() / every

    loss = (torch.where(live, policy + c["kl"] * kl, 0.0).double() * share).sum()
    stats = torch.stack([loss, mean(kl), mean(cut.float()), mean(r), live.sum().double(), (tokens > 0).sum().double()])
    return dict(stats=stats.float(), d_lp=torch.where(live, d * share, 0.0))


# ------------------------------------------------------------------------------------------ work, exact

def work(case):
    kind, size = case["kind"], dict(bf16=2, fp16=2, fp32=4)
    if "norm" in kind:
        rows, n = case["rows"] * case["heads"], case["rows"] * case["heads"] * case["width"]
        x, y, stats = size[case["x"]], size[case["y"]], 4 * rows * (2 if case["norm"] == "layer" else 1)
        small = case["width"] * size[case["w"]] * (2 if case["bias"] else 1)
        forward = n * (x + y) + (n * (x + y) if case["add"] else 0) + stats + small
        back = n * (y + x) + (n * x if case["add"] else 0) + case["width"] * 4 * (2 if case["bias"] else 1)
        if kind == "norm":
            return dict(bytes=forward, flops=6 * n)
        if kind == "norm_grad":
            return dict(bytes=back + n * x + stats + small, flops=12 * n)
        return dict(bytes=forward + back, flops=18 * n)
    if kind == "rope":
        n = case["rows"] * (case["q"] + case["k"])
        return dict(bytes=2 * n * case["dim"] * size[case["type"]] + 4 * case["rows"], flops=3 * n * case["rotary"])
    if "router" in kind:
        T, E, k = case["rows"], case["experts"], case["k"]
        logits, kept, live = T * E * size[case["type"]], T * (4 * k + 4) + 4 * E, T if case["padded"] > 0 else 0
        forward = logits + live + kept + T * 4 * k + 8 * E
        if kind == "router":
            return dict(bytes=forward, flops=6 * T * E)
        if kind == "router_grad":
            return dict(bytes=2 * logits + kept + T * 4 * k, flops=8 * T * E)
        return dict(bytes=forward + T * 4 * k + logits, flops=14 * T * E)
    n = case["rows"]
    live = n - int(n * case["masked"])
    return dict(bytes=8 * n + live * (8 + (4 if case["ref"] else 0)) + (4 * live if case["per_token"] else 4 * case["seqs"]) + 4 * case["seqs"],
                flops=12 * live)


def exact(case, seed):
    kind = case["kind"]
    if "norm" in kind:
        return _exact_norm(case, _prepare_norm(case, seed))
    if kind == "rope":
        return _exact_rope(case, _prepare_rope(case, seed))
    if "router" in kind:
        return _exact_router(case, _prepare_router(case, seed))
    return _exact_policy(case, _prepare_policy(case, seed))


def _exact_norm(case, s):
    got, x, W = {}, s["x"].double(), case["width"]
    forward, back = case["kind"] != "norm_grad", case["kind"] != "norm"
    if forward and case["add"]:
        x = (x + s["add"].double()).to(s["x"].dtype).double()
        got["sum"] = x
    centre = x.sum(-1, keepdim=True) / W if case["norm"] == "layer" else torch.zeros_like(x[..., :1])
    u = x - centre
    r = 1 / ((u * u).sum(-1, keepdim=True) / W + EPS).sqrt()
    if not forward:                                        # the gradient takes the statistics that it is given
        r = s["rstd"].double()[..., None]
        u = x - (s["mean"].double()[..., None] if s["mean"] is not None else 0)
    w = s["weight"].double()
    if forward:
        got["y"] = u * r * w + (s["bias"].double() if case["bias"] else 0)
        got["rstd"] = r[..., 0]
        if case["norm"] == "layer":
            got["mean"] = centre[..., 0]
    if back:
        dy = s["dy"].double()
        n, g = u * r, dy * w
        along = (g * n).sum(-1, keepdim=True) / W
        dx = r * (g - n * along - (g.sum(-1, keepdim=True) / W if case["norm"] == "layer" else 0))
        got["dx"] = dx + s["d_sum"].double() if "d_sum" in s else dx
        got["dw"] = torch.einsum("rw,rw->w", dy.reshape(-1, W), n.reshape(-1, W))
        if case["bias"]:
            got["db"] = dy.reshape(-1, W).sum(0)
    return got


def _exact_rope(case, s):
    got, r = {}, case["rotary"]
    f = []
    for j in range(r // 2):                                # from the formulas, pair by pair
        base = THETA * case["factor"] ** (r / (r - 2)) if case["scaling"] == "base" and r > 2 else THETA
        v = base ** (-2.0 * j / r)
        if case["scaling"] == "linear":
            v /= case["factor"]
        if case["scaling"] == "parts":
            keep = min(1.0, max(0.0, (TRAINED * v / (2 * math.pi) - SLOW) / (FAST - SLOW)))
            v = keep * v + (1 - keep) * v / case["factor"]
        f.append(v)
    angle = torch.outer(s["positions"].double(), torch.tensor(f, dtype=torch.float64, device=DEV))
    turn = torch.polar(torch.full_like(angle, _scale(case)), -angle if case["inverse"] else angle)[:, None]
    for name in ("q", "k"):
        if s[name] is None:
            continue
        t = s[name].double()
        pair = torch.stack(t[..., :r].split(r // 2, dim=-1), -1) if case["layout"] == "half" else t[..., :r].unflatten(-1, (r // 2, 2))
        turned = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        flat = torch.cat([turned[..., 0], turned[..., 1]], -1) if case["layout"] == "half" else turned.flatten(-2)
        got["out_" + name] = torch.cat([flat, t[..., r:]], -1)
    return got


def _exact_router(case, s):
    T, E, k = case["rows"], case["experts"], case["k"]
    z, got = s["logits"].double(), {}
    rows = torch.arange(T, device=DEV) if s["live"] is None else s["live"].nonzero()[:, 0]
    top = z.max(1, keepdim=True).values
    e = (z - top).exp()
    p = e / e.sum(1, keepdim=True)
    lse = top[:, 0] + e.sum(1).log()
    if case["kind"] != "router_grad":
        idx = torch.full((T, k), -1, dtype=torch.int64, device=DEV)
        left = z.clone()
        for i in range(k):                                 # argmax of what is left, the lowest index on ties
            best = left.max(1, keepdim=True).values
            at = (left == best).to(torch.int8).argmax(1)
            idx[:, i] = at
            left[torch.arange(T, device=DEV), at] = -math.inf
        weights = torch.take_along_dim(p, idx, 1)
        if case["renormalise"]:
            weights = weights / weights.sum(1, keepdim=True)
        dead = torch.ones(T, dtype=torch.bool, device=DEV)
        dead[rows] = False
        counts = torch.bincount(idx[rows].flatten(), minlength=E)
        n = max(1, len(rows))
        sums = p[rows].sum(0)
        f, mean = counts.double() / (n * k), sums / n
        losses = torch.stack([E * torch.dot(f, mean), (lse[rows] ** 2).sum() / n])
        idx[dead], weights[dead], kept = -1, 0, lse.clone()
        kept[dead] = 0
        got.update(idx=idx.to(torch.int32), weights=weights, lse=kept, counts=counts.to(torch.int32),
                   offsets=torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32), prob_sums=sums, losses=losses)
        if case["kind"] == "router":
            return got
    else:
        idx, counts = s["idx"].long(), s["counts"].long()
        p = (z - s["lse"].double()[:, None]).exp()         # the gradient takes the lse that it is given
        lse, rows = s["lse"].double(), (idx[:, 0] >= 0).nonzero()[:, 0]
    total = int(counts.sum())
    n = max(1.0, total / k)
    d = torch.zeros(T, E, dtype=torch.float64, device=DEV)
    pr, at, dw = p[rows], idx[rows], s["d_weights"].double()[rows]
    push = (BALANCE * E / n) * counts.double() / max(1, total)
    into = push.expand_as(pr).clone() + 2 * case["z"] / n * lse[rows][:, None]
    # softmax' pulls back every gradient to p; the z loss has the gradient p itself
    dp = push.expand_as(pr).clone()
    sel = torch.take_along_dim(pr, at, 1)
    if case["renormalise"]:
        total_p = sel.sum(1, keepdim=True)
        dsel = dw / total_p - (dw * sel).sum(1, keepdim=True) / total_p ** 2
    else:
        dsel = dw
    dp.scatter_add_(1, at, dsel)
    d[rows] = pr * (dp - (pr * dp).sum(1, keepdim=True)) + pr * (into - push)
    got["d_logits"] = d
    return got


def _exact_policy(case, s):
    lp, old, adv = s["lp"].double(), s["old"].double(), s["adv"].double()
    off, live = s["off"].tolist(), s["targets"] >= 0
    n = case["rows"]
    who = torch.repeat_interleave(torch.arange(case["seqs"], device=DEV), torch.tensor([b - a for a, b in zip(off, off[1:])], device=DEV))
    held = torch.bincount(who[live], minlength=case["seqs"]).double()
    weight = torch.zeros(n, dtype=torch.float64, device=DEV)
    if case["reduce"] == "tokens":
        weight[live] = 1 / max(1.0, float(held.sum()))
    elif case["reduce"] == "sequences":
        weight[live] = (1 / held)[who[live]] / max(1, int((held > 0).sum()))
    else:
        weight[live] = s["scale"]
    a = adv if case["per_token"] else adv[who]
    ratio = (lp - old).exp()
    plain, bounded = ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    cut = bounded < plain
    term = -torch.minimum(plain, bounded)
    d = torch.where(cut, torch.zeros_like(plain), -plain)
    kl = torch.zeros_like(term)
    if s["ref"] is not None:
        x = s["ref"].double() - lp
        kl = x.expm1() - x
        d = d - case["kl"] * x.expm1()
    count = max(1, int(live.sum()))
    stats = [((term + case["kl"] * kl) * weight)[live].sum(), kl[live].sum() / count, cut[live].sum() / count, ratio[live].sum() / count,
             live.sum(), (held > 0).sum()]
    return dict(stats=torch.stack([v.double() for v in stats]), d_lp=d * weight)
