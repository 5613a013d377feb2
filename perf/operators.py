"""The operators of the policy update, as measured: what they compute in plain torch, the calls a user makes
of the framework, and the sizes that stand for their use.

  logprob       log-probability of known tokens under softmax(hidden lm_head^T / T), over a large vocabulary
  logprob_step  the same with its gradient: d hidden and d lm_head of sum_i g_i logp_i
  experts       y_e = x_e w_e^T for rows that are sorted by expert (ragged groups)
  experts_grad  the two gradients of it: dx_e = dy_e w_e and dw_e = dy_e^T x_e
  clip          the norm over all gradients of a list of tensors, and the gradients scaled down to a largest norm

Shapes are those of workloads.py: hidden 2048, vocabulary 151936, 128 experts of 768 (gate and up rows together
1536), 8 experts for each token, prompts of 2048 tokens, 64 sequences; and the tiny model (256, 1024, 8 experts).
"""
import math
import random

import torch

own = False

DEV = "cuda"


def listed():
    return [
        # one token for each of the 64 live sequences: the lm_head is read for few rows
        dict(name="logprob 64 rows", kind="logprob", n=64, hidden=2048, vocab=151936, masked=0.0, temperature=1.0),
        # the response rows of one 2048-token chunk (a quarter is prompt), at the training temperature
        dict(name="logprob chunk", kind="logprob", n=2048, hidden=2048, vocab=151936, masked=0.25, temperature=0.85),
        # a few rows and odd sizes on a small model: launches and latency
        dict(name="logprob_step small", kind="logprob_step", n=37, hidden=264, vocab=1013, masked=0.2, temperature=1.0),
        # a short response on the full vocabulary: gradients of few rows, the whole d lm_head is written
        dict(name="logprob_step short", kind="logprob_step", n=301, hidden=2048, vocab=151936, masked=0.1, temperature=0.85),
        # a packed micro-batch of the update: two prompts of 2048 with their responses, one third masked
        dict(name="logprob_step batch", kind="logprob_step", n=4096, hidden=2048, vocab=151936, masked=0.33, temperature=1.0),
        # one token routed to its eight experts: the smallest call of the expert product
        dict(name="experts one token", kind="experts", rows=8, experts=128, din=2048, dout=1536, skew=0.5, slack=0),
        # 64 sequences x 8 experts at decode: about four rows for each expert, the weights are the work
        dict(name="experts 64 tokens", kind="experts", rows=512, experts=128, din=2048, dout=1536, skew=0.5, slack=0),
        # 8 prompts of 2048 tokens x 8 experts, in a buffer with room behind the last row
        dict(name="experts prompts", kind="experts", rows=131072, experts=128, din=2048, dout=1536, skew=0.3, slack=640),
        # ragged small groups in training: more experts than tiles fill
        dict(name="experts_grad small", kind="experts_grad", rows=1003, experts=32, din=264, dout=520, skew=0.8, slack=5),
        # the down projection's gradients for a micro-batch of 4096 tokens x 8 experts
        dict(name="experts_grad batch", kind="experts_grad", rows=32768, experts=128, din=768, dout=2048, skew=0.5, slack=0),
        # the gradients of one full layer, most of them bf16 and some fp32, each in its flat buffer
        dict(name="clip layer", kind="clip", tensors=9, values=623_000_000, half=0.8, aligned=True, ratio=0.3),
        # the tiny model's gradients at odd places of a flat buffer: the latency of the launches
        dict(name="clip tiny", kind="clip", tensors=12, values=1_100_000, half=0.5, aligned=False, ratio=0.7),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["logprob", "logprob_step", "experts", "experts_grad", "clip"])
    if kind in ("logprob", "logprob_step"):
        n, hidden, vocab = size(1, 4096), 8 * size(32, 256), size(500, 151936)
        return dict(kind=kind, n=n, hidden=hidden, vocab=vocab, masked=round(rng.choice([0.0, rng.uniform(0, 0.8)]), 2),
                    temperature=rng.choice([0.6, 0.85, 1.0]))
    if kind == "clip":
        tensors = size(1, 500)
        return dict(kind=kind, tensors=tensors, values=max(4 * tensors, size(1000, 500_000_000)), half=round(rng.random(), 2),
                    aligned=rng.random() < 0.5, ratio=round(rng.uniform(0.1, 2.0), 2))
    return dict(kind=kind, rows=size(1, 65536 if kind == "experts" else 32768), experts=size(2, 128), din=8 * size(8, 256),
                dout=8 * size(8, 192), skew=round(rng.uniform(0, 1), 2), slack=rng.choice([0, 0, rng.randrange(1, 300)]))


# ----------------------------------------------------------------------------------------------- inputs

def _seeded(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, *shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16) * std).to(dtype)


def _live(case):
    return case["n"] - int(case["n"] * case["masked"])


def _prepare_logprob(case, seed):
    g = _seeded(seed)
    n, H, V = case["n"], case["hidden"], case["vocab"]
    w = _normal(g, V, H, std=0.02)
    targets = torch.randint(V, (n,), generator=g, device=DEV, dtype=torch.int32)
    # a trained model's rows lean towards their token by different amounts: from a guess to near certainty
    lean = torch.rand(n, 1, generator=g, device=DEV) * 20
    row = w[targets.long()].float()
    h = (_normal(g, n, H).float() + lean * row / row.norm(dim=1, keepdim=True)).to(torch.bfloat16)
    masked_rows = torch.randperm(n, generator=g, device=DEV)[: n - _live(case)]
    targets[masked_rows] = -1                                     # prompt and padding rows have no target
    # clipped importance ratio x advantage, over the number of tokens
    d_logp = _normal(g, n, dtype=torch.float32) * torch.rand(n, generator=g, device=DEV) / max(1, _live(case))
    return dict(h=h, w=w, targets=targets, d_logp=d_logp, temperature=case["temperature"])


def _counts(case, seed):
    r = random.Random(int(seed) * 7 + 1)
    E, used = case["experts"], case["rows"]
    if used <= E:                                                 # the experts of one token are distinct
        got = set(r.sample(range(E), used))
        return [1 if e in got else 0 for e in range(E)]
    p = torch.tensor([math.exp(case["skew"] * r.gauss(0, 1)) for _ in range(E)], dtype=torch.float64)
    draws = torch.multinomial(p, used, replacement=True, generator=torch.Generator().manual_seed(int(seed)))
    return torch.bincount(draws, minlength=E).tolist()


def _prepare_experts(case, seed):
    g = _seeded(seed)
    E, K, N, used, total = case["experts"], case["din"], case["dout"], case["rows"], case["rows"] + case["slack"]
    counts = _counts(case, seed)
    off = torch.zeros(E + 1, dtype=torch.int64)
    off[1:] = torch.tensor(counts).cumsum(0)
    s = dict(x=_normal(g, total, K), w=_normal(g, E, N, K, std=0.02), off=off.to(DEV, torch.int32), used=used, most=max(counts))
    if case["kind"] == "experts_grad":
        s["dy"] = _normal(g, total, N, std=0.01)
    return s


def _sizes(case):
    """Numbers of values of the tensors of a gradient list: one large stack, the others smaller and odd."""
    r = random.Random(case["tensors"] * 1_000_003 + case["values"])
    share = [math.exp(2 * r.gauss(0, 1)) for _ in range(case["tensors"])]
    return [max(1, int(case["values"] * v / sum(share))) for v in share]


def _is_half(case, i):
    return (0.61803398875 * (i + 0.5)) % 1 < case["half"]          # spread over the list


def _prepare_clip(case, seed):
    g = _seeded(seed)
    lists, places = {torch.bfloat16: 0, torch.float32: 0}, []
    pad = 128 if case["aligned"] else 1
    for i, n in enumerate(_sizes(case)):
        t = torch.bfloat16 if _is_half(case, i) else torch.float32
        places.append((t, lists[t], n))
        lists[t] += -(-n // pad) * pad
    flat = {t: _normal(g, max(1, n), std=1e-3, dtype=t) for t, n in lists.items()}
    flat[torch.float32].mul_(torch.rand(flat[torch.float32].shape, generator=g, device=DEV))
    out = {t: torch.zeros_like(v) for t, v in flat.items()}
    grads, outs = ([d[t][at:at + n] for t, at, n in places] for d in (flat, out))
    norm = 1e-3 * math.sqrt(sum(n for _, _, n in places))         # about what the values above give
    return dict(flat=flat, out=out, grads=grads, outs=outs, max_norm=case["ratio"] * norm)


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("logprob", "logprob_step"):
        s = _prepare_logprob(case, seed)
    elif kind in ("experts", "experts_grad"):
        s = _prepare_experts(case, seed)
    else:
        s = _prepare_clip(case, seed)
    s["kind"] = kind
    if own:
        s.update(_own_handle(case, s))
    return s


def _own_handle(case, s):
    """The handle and the output tensors that a program keeps beside its inputs."""
    from paper_2511_11373_b200 import binding
    kind = case["kind"]
    if kind in ("logprob", "logprob_step"):
        n = case["n"]
        got = dict(handle=binding.Update(case["hidden"], case["vocab"], n, device=DEV),
                   logp=torch.empty(n, device=DEV), lse=torch.empty(n, device=DEV))
        if kind == "logprob_step":
            got.update(d_h=torch.empty_like(s["h"]), d_w=torch.empty_like(s["w"]))
        return got
    if kind == "clip":
        return dict(handle=binding.GradList(s["grads"], s["outs"]), norm=torch.empty(1, device=DEV))
    got = dict(handle=binding.Update(0, 0, 0, device=DEV))
    total, E = s["x"].shape[0], case["experts"]
    if kind == "experts":
        got.update(y=torch.zeros(total, case["dout"], dtype=torch.bfloat16, device=DEV))
    else:
        got.update(dx=torch.zeros_like(s["x"]), dw=torch.empty_like(s["w"]))
    return got


# ------------------------------------------------------------------------------------------------- run

def run(s):
    return _run_own(s) if own else _PLAIN[s["kind"]](s)


def _run_own(s):
    from paper_2511_11373_b200 import binding
    kind, u = s["kind"], s["handle"]
    if kind in ("logprob", "logprob_step"):
        st = binding.mars_logprob(u, s["h"], s["w"], s["targets"], s["temperature"], s["logp"], s["lse"])
        if kind == "logprob":
            got = dict(logp=s["logp"])
        else:
            st = st or binding.mars_logprob_grad(u, s["h"], s["w"], s["targets"], s["temperature"], s["lse"], s["d_logp"],
                                                 s["d_h"], s["d_w"], logprobs=s["logp"])
            got = dict(logp=s["logp"], d_h=s["d_h"], d_w=s["d_w"])
    elif kind == "experts":
        st = binding.mars_expert_matmul(u, s["x"], s["off"], s["w"], s["y"])
        got = dict(y=s["y"])
    elif kind == "experts_grad":
        st = binding.mars_expert_matmul_dx(u, s["dy"], s["off"], s["w"], s["dx"])
        st = st or binding.mars_expert_matmul_dw(u, s["dy"], s["x"], s["off"], s["dw"])
        got = dict(dx=s["dx"], dw=s["dw"])
    else:
        st = binding.mars_grads_clip(u, s["max_norm"], s["norm"])
        got = dict(norm=s["norm"], half=s["out"][torch.bfloat16], full=s["out"][torch.float32])
    if st:
        raise RuntimeError("status %d" % st)
    return got


def _plain_logprob(s):
    z = s["h"].float() @ s["w"].float().T / s["temperature"]
    lse = torch.logsumexp(z, dim=1)
    live = s["targets"] >= 0
    at = s["targets"].clamp(min=0).long()[:, None]
    logp = torch.where(live, z.gather(1, at)[:, 0] - lse, 0.0)
    if s["kind"] == "logprob":
        return dict(logp=logp)
    g = torch.where(live, s["d_logp"], 0.0) / s["temperature"]
    d = torch.exp(z - lse[:, None]).mul_(-g[:, None])
    # 1 - p of the token itself, where p is near 1, from the sum of the others
    rest = -(torch.expm1(logp)) * g
    d.scatter_(1, at, rest[:, None])
    return dict(logp=logp, d_h=(d @ s["w"].float()).to(torch.bfloat16), d_w=(d.T @ s["h"].float()).to(torch.bfloat16))


def _places(s):
    """Expert and place in its group of every used row."""
    i = torch.arange(s["used"], device=DEV)
    e = torch.searchsorted(s["off"][1:].contiguous(), i.to(torch.int32), right=True)
    return e, i - s["off"].long()[e]


def _padded(s, rows):
    e, at = _places(s)
    got = torch.zeros(s["w"].shape[0], s["most"], rows.shape[1], device=DEV)
    got[e, at] = rows[: s["used"]].float()
    return got


def _ragged(s, padded, like):
    e, at = _places(s)
    got = torch.zeros(like, padded.shape[2], dtype=torch.bfloat16, device=DEV)
    got[: s["used"]] = padded[e, at].to(torch.bfloat16)
    return got


def _plain_experts(s):
    return dict(y=_ragged(s, torch.bmm(_padded(s, s["x"]), s["w"].float().transpose(1, 2)), s["x"].shape[0]))


def _plain_experts_grad(s):
    dy = _padded(s, s["dy"])
    dx = _ragged(s, torch.bmm(dy, s["w"].float()), s["x"].shape[0])
    return dict(dx=dx, dw=torch.bmm(dy.transpose(1, 2), _padded(s, s["x"])).to(torch.bfloat16))


def _plain_clip(s):
    norm = torch.stack([t.double().square().sum() for t in s["grads"]]).sum().sqrt()
    scale = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0).float()
    [o.copy_(t.float() * scale) for t, o in zip(s["grads"], s["outs"])]
    return dict(norm=norm.float().reshape(1), half=s["out"][torch.bfloat16], full=s["out"][torch.float32])


_PLAIN = dict(logprob=_plain_logprob, logprob_step=_plain_logprob, experts=_plain_experts, experts_grad=_plain_experts_grad,
              clip=_plain_clip)


# ------------------------------------------------------------------------------------------ work, exact

def work(case):
    kind = case["kind"]
    if kind in ("logprob", "logprob_step"):
        live, H, V = _live(case), case["hidden"], case["vocab"]
        read = 2 * live * H + 2 * V * H + 4 * case["n"]
        if kind == "logprob":
            return dict(bytes=read + 4 * case["n"], flops=2 * live * H * V)
        # the logits once and the two products of the gradient
        return dict(bytes=read + 8 * case["n"] + 2 * case["n"] * H + 2 * V * H, flops=6 * live * H * V)
    if kind == "clip":
        n = sum((2 if _is_half(case, i) else 4) * v for i, v in enumerate(_sizes(case)))
        return dict(bytes=2 * n, flops=3 * sum(_sizes(case)))
    rows, E, K, N = case["rows"], case["experts"], case["din"], case["dout"]
    weights = 2 * min(rows, E) * K * N
    if kind == "experts":
        return dict(bytes=2 * rows * (K + N) + weights + 4 * E, flops=2 * rows * K * N)
    return dict(bytes=2 * rows * (K + N) + 2 * rows * K + weights + 2 * E * K * N + 4 * E, flops=4 * rows * K * N)


def exact(case, seed):
    s = (_prepare_logprob if "logprob" in case["kind"] else _prepare_clip if case["kind"] == "clip" else _prepare_experts)(case, seed)
    return {"clip": _exact_clip, "experts": _exact_experts, "experts_grad": _exact_experts}.get(case["kind"], _exact_logprob)(case, s)


def _exact_logprob(case, s):
    h, w, T = s["h"].double(), s["w"].double(), case["temperature"]
    n, V = h.shape[0], w.shape[0]
    logp = torch.zeros(n, dtype=torch.float64, device=DEV)
    grad = case["kind"] == "logprob_step"
    d_h, d_w = torch.zeros_like(h), torch.zeros_like(w) if grad else None
    rows = [i for i, t in enumerate(s["targets"].tolist()) if t >= 0]
    for at in range(0, len(rows), 512):                           # 512 live rows at a time
        r = torch.tensor(rows[at:at + 512], device=DEV)
        t = s["targets"][r].long()
        me = torch.arange(len(r), device=DEV)
        z = torch.mm(h[r], w.t()).div_(T)
        z -= z.max(dim=1, keepdim=True).values
        e = z.exp()
        total = e.sum(dim=1)
        logp[r] = z[me, t] - total.log()
        if grad:
            p = e / total[:, None]
            others = e.clone()
            others[me, t] = 0
            p[me, t] = -others.sum(dim=1) / total                 # p - 1 without cancellation
            p *= -(s["d_logp"][r].double() / T)[:, None]
            d_h[r] = torch.mm(p, w)
            d_w += torch.mm(p.t(), h[r])
    return dict(logp=logp, d_h=d_h, d_w=d_w) if grad else dict(logp=logp)


def _exact_experts(case, s):
    off = s["off"].tolist()
    total, E, K, N = s["x"].shape[0], case["experts"], case["din"], case["dout"]
    y, dx = torch.zeros(total, N, dtype=torch.float64, device=DEV), torch.zeros(total, K, dtype=torch.float64, device=DEV)
    dw = torch.zeros(E, N, K, dtype=torch.float64, device=DEV) if "dy" in s else None
    for e in range(E):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        we, xe = s["w"][e].double(), s["x"][a:b].double()
        if "dy" in s:
            dye = s["dy"][a:b].double()
            dx[a:b], dw[e] = dye @ we, dye.t() @ xe
        else:
            y[a:b] = xe @ we.t()
    return dict(dx=dx, dw=dw) if "dy" in s else dict(y=y)


def _exact_clip(case, s):
    total = math.fsum(float((t.double() ** 2).sum()) for t in s["grads"])
    norm = math.sqrt(total)
    scale = min(1.0, s["max_norm"] / (norm + 1e-6))
    got = {t: torch.zeros(v.shape, dtype=torch.float64, device=DEV) for t, v in s["flat"].items()}
    for t, g in got.items():
        base = s["flat"][t].data_ptr()
        for x in s["grads"]:
            if x.dtype == t:
                at = (x.data_ptr() - base) // x.element_size()
                g[at:at + x.numel()] = x.double() * scale
    return dict(norm=torch.tensor([norm], dtype=torch.float64), half=got[torch.bfloat16], full=got[torch.float32])
