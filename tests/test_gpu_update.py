"""Policy-update operators on the GPU against plain 64-bit forms: log-probability with its gradient, expert products with
theirs, gradient norm and clipping.

Tolerances are bounds from the arithmetic, evaluated on each test's own inputs.  u(t) = half a step of type t
(bf16 2^-8, fp16 2^-11, fp32 2^-24, relative to the value).  A tensor-core sum over K products of bf16 values is exact in
each product and adds in fp32, 16 products at a time, by at most one fp32 step (2^-23) of the running sum for each
addition: |error| <= (K / 16 + 16) 2^-23 sum |a| |b|.
"""
import math

import pytest
import torch

from paper_2511_11373_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(torch.bfloat16)


def sum_error(K):
    return (K / 16 + 16) * 2.0 ** -23


def worst(got, want, tol):
    """Largest error in units of its tolerance (NaN counts as infinite)."""
    e = ((got.double() - want).abs() / tol.clamp_min(1e-300))
    e = torch.where((got.double() == want), torch.zeros_like(e), e)
    return float(torch.nan_to_num(e, nan=math.inf).max()) if e.numel() else 0.0


# ------------------------------------------------------------------------------------------ log-prob

def logprob_reference(h, w, targets, T, g=None):
    """logp, lse, and with g the gradients, in fp64; rows without a target are 0."""
    hd, wd, live = h.double(), w.double(), targets >= 0
    hd = torch.where(live[:, None], hd, 0.0)
    z = hd @ wd.t() / T
    lse = torch.logsumexp(z, dim=1)
    at = targets.clamp(min=0).long()
    logp = torch.where(live, z[torch.arange(len(at)), at] - lse, 0.0)
    out = dict(logp=logp, lse=torch.where(live, lse, 0.0))
    # error of a logit, and of log-probs made of two of them: |h| |w|^T is the sum of absolute products
    scale = (hd.abs() @ wd.abs().t()).max(dim=1).values / T if z.numel() else torch.zeros(len(at), device=DEV)
    K = h.shape[1]
    # + rounding of the result, of the running sums (2^-22 relative each over V / 32 joins) and of exp2 / log
    out["tol"] = 2 * sum_error(K) * scale + 2.0 ** -22 * (16 + lse.abs()) + 2.0 ** -23 * math.sqrt(w.shape[0])
    if g is not None:
        gd = torch.where(live, g.double(), 0.0) / T
        d = -torch.exp(z - lse[:, None]) * gd[:, None]
        d[torch.arange(len(at)), at] += gd
        out["d_h"], out["d_w"] = d @ wd, d.t() @ hd
        # an entry of d is off by its rounding to bf16 and by exp of an exponent that is off by the logit's error and lse's
        rel = U[torch.bfloat16] * 1.01 + 2 * out["tol"][:, None]
        # (1 - p of the target: its error is that of the exponent times p, absolute)
        da = d.abs() * rel + (2 * out["tol"] * gd.abs())[:, None] * torch.exp(z - lse[:, None])
        V, n = w.shape[0], h.shape[0]
        out["tol_h"] = da @ wd.abs() + sum_error(V) * (d.abs() @ wd.abs())
        out["tol_w"] = da.t() @ hd.abs() + sum_error(n) * (d.abs().t() @ hd.abs())
    return out


def logprob_case(n, H, V, T, masked=0.0, seed=0, pad=0, lean=6.0):
    g = gen(seed)
    w = normal(g, V, H, std=0.05)
    targets = torch.randint(V, (n,), generator=g, device=DEV, dtype=torch.int32)
    rows = w[targets.long()].float()
    h = normal(g, n, H + pad)
    h[:, :H] = (h[:, :H].float() + lean * torch.rand(n, 1, generator=g, device=DEV) * rows / rows.norm(dim=1, keepdim=True).clamp_min(1e-6))
    h = h[:, :H]
    off = torch.rand(n, generator=g, device=DEV) < masked
    targets[off] = -1
    d = torch.randn(n, generator=g, device=DEV)
    return h, w, targets, d


def run_logprob(u, h, w, targets, T, d=None, dtype=torch.bfloat16, base=None, stream=None):
    n = h.shape[0]
    logp, lse = (torch.full((n,), 77.0, device=DEV) for _ in range(2))
    assert binding.mars_logprob(u, h, w, targets, T, logp, lse, stream=stream) == 0
    out = dict(logp=logp, lse=lse)
    if d is not None:
        out["d_h"] = torch.full((n, h.shape[1]), 77.0, dtype=torch.bfloat16, device=DEV)
        out["d_w"] = torch.full(w.shape, 77.0, dtype=dtype, device=DEV) if base is None else base.clone()
        assert binding.mars_logprob_grad(u, h, w, targets, T, lse, d, out["d_h"], out["d_w"], accumulate=base is not None,
                                         stream=stream) == 0
    return out


def check_logprob(got, ref, base=None):
    u = U[torch.bfloat16]
    assert worst(got["logp"], ref["logp"], ref["tol"]) <= 1
    assert worst(got["lse"], ref["lse"], ref["tol"]) <= 1
    if "d_h" in got:
        assert worst(got["d_h"], ref["d_h"], ref["tol_h"] + u * (ref["d_h"].abs() + ref["tol_h"]) + 1e-38) <= 1
        want = ref["d_w"] + (0 if base is None else base.double())
        r = U[got["d_w"].dtype]
        assert worst(got["d_w"], want, ref["tol_w"] + r * (want.abs() + ref["tol_w"]) + 2.0 ** -23 * want.abs() + 1e-38) <= 1


@pytest.mark.parametrize("n,H,V,T,masked,pad", [
    (1, 8, 1, 1.0, 0.0, 0), (1, 64, 7, 1.0, 0.0, 0), (2, 72, 257, 0.7, 0.0, 8), (4, 256, 1024, 1.0, 0.0, 0), (37, 264, 1013, 0.85, 0.3, 16),
    (64, 128, 512, 1.0, 0.0, 0), (65, 136, 513, 1.0, 0.5, 0), (128, 200, 2000, 0.6, 0.1, 0), (129, 256, 255, 1.0, 0.2, 0),
    (255, 64, 4097, 1.3, 0.9, 0), (300, 520, 3001, 0.85, 0.2, 24), (513, 328, 2049, 1.0, 0.0, 0)])
def test_logprob_and_gradient_match_the_formula(n, H, V, T, masked, pad):
    h, w, targets, d = logprob_case(n, H, V, T, masked, seed=n + V, pad=pad)
    u = binding.Update(H, V, n, device=DEV)
    got = run_logprob(u, h, w, targets, T, d)
    assert u.poll_status() == 0
    check_logprob(got, logprob_reference(h, w, targets, T, d))
    dead = targets < 0
    assert (got["logp"][dead] == 0).all() and (got["lse"][dead] == 0).all() and (got["d_h"][dead] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_of_lm_head_in_both_types_and_accumulated(dtype):
    h, w, targets, d = logprob_case(150, 136, 700, 1.0, 0.2, seed=5)
    u = binding.Update(136, 700, 400, device=DEV)                # a handle for more rows than the call has
    base = (torch.randn(700, 136, generator=gen(1), device=DEV) * 0.1).to(dtype)
    ref = logprob_reference(h, w, targets, 1.0, d)
    check_logprob(run_logprob(u, h, w, targets, 1.0, d, dtype=dtype), ref)
    check_logprob(run_logprob(u, h, w, targets, 1.0, d, base=base), ref, base=base)


def test_rows_without_a_target_or_weight_may_hold_anything():
    h, w, targets, d = logprob_case(140, 128, 600, 1.0, 0.4, seed=8)
    d[::7] = 0.0
    ref = logprob_reference(h, w, targets, 1.0, d)
    u = binding.Update(128, 600, 140, device=DEV)
    clean = run_logprob(u, h, w, targets, 1.0, d)
    check_logprob(clean, ref)
    bad = h.clone()
    dead = targets < 0
    bad[dead] = float("nan")
    bad[dead.nonzero()[:3, 0]] = float("inf")
    d2 = d.clone()
    d2[dead] = float("nan")
    got = run_logprob(u, bad, w, targets, 1.0, d2)
    for k in clean:
        assert torch.equal(clean[k], got[k]), k
    # weight 0: no part in the gradient, whatever the row holds
    lse = clean["lse"].clone()
    bad2 = h.clone()
    bad2[d == 0] = float("nan")
    lse[d == 0] = float("nan")
    d_h, d_w = torch.empty_like(clean["d_h"]), torch.empty_like(clean["d_w"])
    assert binding.mars_logprob_grad(u, bad2, w, targets, 1.0, lse, d, d_h, d_w) == 0
    assert torch.equal(d_h, clean["d_h"]) and torch.equal(d_w, clean["d_w"])
    assert (d_h[d == 0] == 0).all()


@pytest.mark.parametrize("n", [1, 130])
def test_no_live_row(n):
    h, w, targets, d = logprob_case(n, 64, 300, 1.0, seed=3)
    targets.fill_(-1)
    u = binding.Update(64, 300, n, device=DEV)
    got = run_logprob(u, h, w, targets, 1.0, d)
    assert all((v == 0).all() for v in got.values())
    base = torch.randn(300, 64, device=DEV)
    got = run_logprob(u, h, w, targets, 1.0, d, base=base)
    assert torch.equal(got["d_w"], base)


def test_zero_rows():
    w = normal(gen(1), 300, 64)
    u = binding.Update(64, 300, 10, device=DEV)
    e = torch.empty(0, device=DEV)
    h, t = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    assert binding.mars_logprob(u, h, w, t, 1.0, e, e) == 0
    d_w = torch.ones_like(w)
    assert binding.mars_logprob_grad(u, h, w, t, 1.0, e, e, h, d_w, accumulate=True) == 0
    assert (d_w == 1).all()
    assert binding.mars_logprob_grad(u, h, w, t, 1.0, e, e, h, d_w) == 0
    assert (d_w == 0).all()


def test_confident_and_extreme_rows():
    """Probabilities near 1 (1 - p without cancellation), equal logits, large logits and a target that underflows."""
    g = gen(4)
    V, H = 900, 64
    w = normal(g, V, H)
    t = torch.tensor([3, 5, 899, 0, 17], dtype=torch.int32, device=DEV)
    h = normal(g, 5, H)
    h[0] = (w[3].float() * 0.25).bfloat16()                       # p close to 1
    h[1] = 0                                                      # uniform
    h[2] = (w[899].float() * 40).bfloat16()                       # logits in the thousands
    h[3] = (w[0].float() * -8).bfloat16()                         # the target far below the others
    d = torch.tensor([1.0, -2.0, 0.5, 1e-3, 1e4], device=DEV)
    u = binding.Update(H, V, 5, device=DEV)
    check_logprob(run_logprob(u, h, w, t, 1.0, d), logprob_reference(h, w, t, 1.0, d))


@pytest.mark.parametrize("n", [64, 200])
@pytest.mark.parametrize("T", [1.0, 0.85, 0.6])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_confident_rows_keep_the_relative_accuracy_of_1_minus_p(n, T, dtype):
    """1 - p of the targets from 1e-2 down to 1e-9, each row weighted by its 1 / (1 - p): with the log-probs at hand every
    entry of d, the target's included, is right to the error of an exponent and its rounding."""
    H, V = 64, 900
    g = gen(71)
    w = normal(g, V, H)
    targets = torch.randperm(V, generator=g, device=DEV)[:n].to(torch.int32)
    at, me = targets.long(), torch.arange(n, device=DEV)
    rows = w[at].double()
    h = (rows * (torch.linspace(12.0, 36.0, n, device=DEV)[:, None] * T / rows.square().sum(1, keepdim=True))).bfloat16()
    hd, wd = h.double(), w.double()
    z = hd @ wd.t() / T
    e = torch.exp(z - z[me, at][:, None])
    e[me, at] = 0
    rest = e.sum(1)
    one_p = rest / (1 + rest)
    assert 1e-11 < float(one_p.min()) < 1e-7 and 5e-3 < float(one_p.max()) < 5e-2
    weight = (1 / one_p).float()
    u = binding.Update(H, V, n, device=DEV)
    logp, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    assert binding.mars_logprob(u, h, w, targets, T, logp, lse) == 0
    d_h, d_w = torch.empty_like(h), torch.empty(V, H, dtype=dtype, device=DEV)
    assert binding.mars_logprob_grad(u, h, w, targets, T, lse, weight, d_h, d_w, logprobs=logp) == 0
    d = -e / (1 + rest)[:, None]
    d[me, at] = one_p
    d *= weight.double()[:, None] / T
    # an entry is off by its exponent (two logits and lse) and by its rounding: one bf16 row, or two up to 128 rows
    scale = (hd.abs() @ wd.abs().t()).max(dim=1).values / T
    rel = 2 * (2 * sum_error(H) * scale + 2.0 ** -22 * (16 + z[me, at].abs()) + 2.0 ** -23 * math.sqrt(V))
    assert float(rel.max()) < 1e-3
    da = d.abs() * (rel + (2.0 ** -16 if n <= 128 else 1.01 * 2.0 ** -8))[:, None]
    for got, want, tol in ((d_h, d @ wd, da @ wd.abs() + sum_error(V) * (d.abs() @ wd.abs())),
                           (d_w, d.t() @ hd, da.t() @ hd.abs() + sum_error(n) * (d.abs().t() @ hd.abs()))):
        check_rounded(got, want, tol)


@pytest.mark.parametrize("T", [1.0, 0.85])
def test_a_certain_token_has_no_gradient(T):
    """Logits in the thousands, p = 1 in fp64: nothing is left, whatever the rounding of lse."""
    g = gen(72)
    w = normal(g, 300, 64)
    targets = torch.arange(20, device=DEV, dtype=torch.int32)
    h = (w[:20].float() * 40).bfloat16()
    u = binding.Update(64, 300, 20, device=DEV)
    logp, lse = torch.empty(20, device=DEV), torch.empty(20, device=DEV)
    assert binding.mars_logprob(u, h, w, targets, T, logp, lse) == 0
    assert (logp == 0).all()
    d_h, d_w = torch.ones_like(h), torch.ones_like(w)
    assert binding.mars_logprob_grad(u, h, w, targets, T, lse, torch.ones(20, device=DEV), d_h, d_w, logprobs=logp) == 0
    assert (d_h == 0).all() and (d_w == 0).all()
    bad = binding.lib().mars_logprob_grad_lp                    # the log-probs are an input like the others
    args = [u.handle, None, 20, h.data_ptr(), 64, w.data_ptr(), targets.data_ptr(), T, logp.data_ptr() + 2, lse.data_ptr(), lse.data_ptr(),
            d_h.data_ptr(), 64, d_w.data_ptr(), 1, 0]
    assert bad(*args) == 1
    args[8] = d_h.data_ptr()
    assert bad(*args) == 1
    with pytest.raises(ValueError):
        binding.mars_logprob_grad(u, h, w, targets, T, lse, lse, d_h, d_w, logprobs=logp.double())


def test_target_beyond_the_vocabulary_is_reported_and_left_out():
    h, w, targets, d = logprob_case(20, 64, 300, 1.0, seed=9)
    targets[4] = 300
    targets[9] = 2 ** 31 - 1
    u = binding.Update(64, 300, 20, device=DEV)
    got = run_logprob(u, h, w, targets, 1.0, d)
    assert u.poll_status() == 7 and u.poll_status() == 0
    targets[4] = targets[9] = -1
    check_logprob(got, logprob_reference(h, w, targets, 1.0, d))


@pytest.mark.parametrize("n,V", [(40, 33), (300, 777)])
def test_gradient_against_differences(n, V):
    """sum_i g_i logp_i at h +- e dir and w +- e dir in fp64, against the kernel's gradient along dir."""
    H, T = 72, 0.85
    h, w, targets, d = logprob_case(n, H, V, T, 0.2, seed=n)
    u = binding.Update(H, V, n, device=DEV)
    got = run_logprob(u, h, w, targets, T, d, dtype=torch.float32)
    ref = logprob_reference(h, w, targets, T, d)
    live, at = targets >= 0, targets.clamp(min=0).long()

    def loss(hd, wd):
        z = hd @ wd.t() / T
        lp = z[torch.arange(n), at] - torch.logsumexp(z, dim=1)
        return float((torch.where(live, d.double(), 0.0) * lp).sum())

    g, e = gen(77), 1e-5
    for of in ("d_h", "d_w"):
        for _ in range(4):
            x = h.double() if of == "d_h" else w.double()
            v = torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float64)
            if of == "d_h":
                diff = (loss(x + e * v, w.double()) - loss(x - e * v, w.double())) / (2 * e)
                tol = float(((ref["tol_h"] + U[torch.bfloat16] * ref["d_h"].abs()) * v.abs()).sum())
            else:
                diff = (loss(h.double(), x + e * v) - loss(h.double(), x - e * v)) / (2 * e)
                tol = float((ref["tol_w"] * v.abs()).sum())
            assert abs(float((got[of].double() * v).sum()) - diff) <= tol + 1e-6 * abs(diff) + 1e-5


def test_several_vocabulary_pieces():
    """A large row count makes the pieces narrow: five pieces, the last one ragged."""
    n, H, V = 33000, 64, 33333
    u = binding.Update(H, V, n, device=DEV)
    h, w, targets, d = logprob_case(n, H, V, 1.0, 0.99, seed=2)
    targets[0], targets[1], targets[n - 1] = 6911, 6912, V - 1
    got = run_logprob(u, h, w, targets, 1.0, d)
    live = targets >= 0
    ref = logprob_reference(h[live], w, targets[live], 1.0, d[live])
    check_logprob(dict(logp=got["logp"][live], lse=got["lse"][live], d_h=got["d_h"][live], d_w=got["d_w"]), ref)
    assert (got["d_h"][~live] == 0).all()


def test_the_largest_row_count():
    n, H, V = 1 << 20, 16, 300
    u = binding.Update(H, V, n, device=DEV)
    h, w, targets, d = logprob_case(n, H, V, 1.0, 0.3, seed=3)
    got = run_logprob(u, h, w, targets, 0.85, d, dtype=torch.float32)
    assert u.poll_status() == 0
    ref = logprob_reference(h, w, targets, 0.85, d)
    check_logprob(got, ref)


def test_full_vocabulary_rows():
    n, H, V = 70, 2048, 151936
    h, w, targets, d = logprob_case(n, H, V, 1.0, 0.1, seed=6)
    u = binding.Update(H, V, n, device=DEV)
    check_logprob(run_logprob(u, h, w, targets, 1.0, d), logprob_reference(h, w, targets, 1.0, d))


def test_same_bits_on_another_stream_and_in_a_graph():
    h, w, targets, d = logprob_case(290, 128, 1500, 1.0, 0.2, seed=12)
    u = binding.Update(128, 1500, 290, device=DEV)
    first = run_logprob(u, h, w, targets, 1.0, d)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = run_logprob(u, h, w, targets, 1.0, d)
    s.synchronize()
    for k in first:
        assert torch.equal(first[k], again[k]), k
    # captured once, replayed on new inputs in the same memory
    graph = torch.cuda.CUDAGraph()
    out = dict(logp=torch.zeros(290, device=DEV), lse=torch.zeros(290, device=DEV), d_h=torch.zeros_like(first["d_h"]),
               d_w=torch.zeros_like(first["d_w"]))
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        assert binding.mars_logprob(u, h, w, targets, 1.0, out["logp"], out["lse"]) == 0
        assert binding.mars_logprob_grad(u, h, w, targets, 1.0, out["lse"], d, out["d_h"], out["d_w"]) == 0
    graph.replay()
    torch.cuda.synchronize()
    for k in first:
        assert torch.equal(first[k], out[k]), k
    targets.copy_(torch.where(targets < 0, 5, -1))                # other live rows, more of them
    targets[100:] = 3
    graph.replay()
    torch.cuda.synchronize()
    check_logprob(out, logprob_reference(h, w, targets, 1.0, d))
    assert u.poll_status() == 0


def test_logprob_refusals():
    h, w, targets, d = logprob_case(8, 64, 100, 1.0, seed=1)
    u = binding.Update(64, 100, 8, device=DEV)
    lp, lse = torch.empty(8, device=DEV), torch.empty(8, device=DEV)
    d_h, d_w = torch.full_like(h, 3.0), torch.full_like(w, 3.0)
    for T in (0.0, -1.0, float("nan"), float("inf")):
        assert binding.mars_logprob(u, h, w, targets, T, lp, lse) == 1
        assert binding.mars_logprob_grad(u, h, w, targets, T, lse, d, d_h, d_w) == 1
    assert binding.mars_logprob(u, h, w, targets, 1.0, lp, lp) == 1                     # outputs on top of each other
    assert binding.mars_logprob_grad(u, h, w, targets, 1.0, lse, d, h, d_w) == 1        # an output on an input
    assert binding.mars_logprob_grad(u, h, w, targets, 1.0, lse, d, d_h, w) == 1
    big = torch.zeros(9, 64, dtype=torch.bfloat16, device=DEV)
    t9, f9 = torch.zeros(9, dtype=torch.int32, device=DEV), torch.empty(9, device=DEV)
    assert binding.mars_logprob(u, big, w, t9, 1.0, f9, torch.empty(9, device=DEV)) == 1     # more rows than the handle has
    odd = torch.zeros(8, 65, dtype=torch.bfloat16, device=DEV)
    assert binding.mars_logprob(u, odd[:, :64], w, targets, 1.0, lp, lse) == 1          # row stride off 8 elements
    off = torch.zeros(8 * 72 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(8, 72)
    assert binding.mars_logprob(u, off[:, :64], w, targets, 1.0, lp, lse) == 1          # off its alignment
    e = binding.Update(0, 0, 0, device=DEV)                                             # a handle without an lm_head
    with pytest.raises(ValueError):
        binding.mars_logprob(e, h, w, targets, 1.0, lp, lse)
    assert (d_h == 3).all() and (d_w == 3).all() and u.poll_status() == 0


def test_a_temperature_without_a_reciprocal_is_refused():
    h, w, targets, _ = logprob_case(8, 64, 100, 1.0, seed=1)
    u = binding.Update(64, 100, 8, device=DEV)
    lp, lse = torch.full((8,), 3.0, device=DEV), torch.empty(8, device=DEV)
    assert binding.mars_logprob(u, h, w, targets, 2.0 ** -129, lp, lse) == 1           # 1 / T is an infinity in fp32
    torch.cuda.synchronize()
    assert (lp == 3).all()
    assert binding.mars_logprob(u, h, w, targets, 2.0 ** -120, lp, lse) == 0           # and here it is not


def test_the_smallest_temperatures():
    """log2(e) / T, the factor that the kernels use, leaves fp32 before 1 / T does."""
    h, w, targets, d = logprob_case(8, 64, 100, 1.0, seed=1)
    h = (h.float() * 2.0 ** -40).bfloat16()                       # logits that stay finite when they are divided by T
    u = binding.Update(64, 100, 8, device=DEV)
    lp, lse = torch.full((8,), 3.0, device=DEV), torch.full((8,), 3.0, device=DEV)
    d_h, d_w = torch.full_like(h, 3.0), torch.full_like(w, 3.0)
    for T in (1.1 * 2.0 ** -128, 1.4 * 2.0 ** -128):
        assert binding.mars_logprob(u, h, w, targets, T, lp, lse) == 1
        assert binding.mars_logprob_grad(u, h, w, targets, T, lse, d, d_h, d_w) == 1
    torch.cuda.synchronize()
    assert all((t == 3).all() for t in (lp, lse, d_h, d_w))
    for T in (1.5 * 2.0 ** -128, 2.0 ** -120):
        got = run_logprob(u, h, w, targets, T)
        assert torch.isfinite(got["logp"]).all()
        check_logprob(got, logprob_reference(h, w, targets, T))


def gradient_error(n, V=4000, H=128):
    """2-norm error of an fp32 d_lm_head relative to its size, rows of nearly uniform p (nothing but roundings of d)."""
    g = gen(91)
    w, h = normal(g, V, H, std=0.05), normal(g, n, H)
    targets = torch.randint(V, (n,), generator=g, device=DEV, dtype=torch.int32)
    d = torch.randn(n, generator=g, device=DEV)
    u = binding.Update(H, V, n, device=DEV)
    got = run_logprob(u, h, w, targets, 1.0, d, dtype=torch.float32)["d_w"].double()
    z = h.double() @ w.double().t()
    dz = -torch.softmax(z, dim=1)
    dz[torch.arange(n), targets.long()] += 1
    want = (dz * d.double()[:, None]).t() @ h.double()
    other = torch.ones(V, dtype=torch.bool, device=DEV)
    other[targets.long()] = False                                 # rows of p alone: entries of one size
    return float((got[other] - want[other]).norm() / want[other].norm())


def test_the_second_bf16_row_of_short_calls_counts():
    """Up to 128 rows d is held in two bf16 rows, together within 2^-16 of an entry; beyond in one, within 2^-8 of it, which is
    2^-8 / sqrt(7) in the 2-norm.  The logits' own errors (2e-6) are below both."""
    assert gradient_error(128) < 2.0 ** -14
    assert gradient_error(64) < 2.0 ** -14
    assert 2.0 ** -11.5 < gradient_error(129) < 2.0 ** -9


@pytest.mark.parametrize("n", [700, 1030])
def test_log_probs_of_more_rows_than_a_block_of_tiles(n):
    """At 16384 wide 1024 rows (four tiles) stay in L2 while the lm_head passes; at 65536 wide 256 do, one tile."""
    for H, V in ((16384, 800), (65536, 300)):
        h, w, targets, d = logprob_case(n, H, V, 1.0, 0.0, seed=n)
        h, w = (h.float() / 16).bfloat16(), (w.float() / 4).bfloat16()
        u = binding.Update(H, V, n, device=DEV)
        check_logprob(run_logprob(u, h, w, targets, 0.85, d), logprob_reference(h, w, targets, 0.85, d))


def test_lm_head_beyond_32_bit_offsets():
    """2.5e9 entries: the target rows in the last and first parts of the matrix, against fp64 on the rows that count."""
    n, H, V = 3, 8192, 300001
    g = gen(31)
    w = torch.empty(V, H, dtype=torch.bfloat16, device=DEV)
    w.normal_(std=0.01, generator=g)
    h = normal(g, n, H)
    targets = torch.tensor([V - 1, 262145, 5], dtype=torch.int32, device=DEV)
    d = torch.tensor([1.0, -0.5, 2.0], device=DEV)
    u = binding.Update(H, V, n, device=DEV)
    got = run_logprob(u, h, w, targets, 1.0, d)
    z = torch.cat([h.double() @ w[a:a + 50000].double().t() for a in range(0, V, 50000)], dim=1)
    lse = torch.logsumexp(z, dim=1)
    at = targets.long()
    logp = z[torch.arange(n), at] - lse
    scale = max(float((h.double().abs() @ w[a:a + 50000].double().abs().t()).max()) for a in range(0, V, 50000))
    tol = 2 * sum_error(H) * scale + 2.0 ** -22 * 32 + 2.0 ** -23 * math.sqrt(V)
    assert (got["logp"].double() - logp).abs().max() <= tol
    rows = torch.tensor([0, 5, 262143, 262144, 262145, V - 2, V - 1], device=DEV)
    dz = -torch.exp(z[:, rows] - lse[:, None]) * d.double()[:, None]
    for i in range(n):
        dz[i] += torch.where(rows == at[i], d.double()[i], 0.0)
    want = dz.t() @ h.double()
    size = (dz.abs() + 2 * tol).t() @ h.double().abs()
    assert ((got["d_w"][rows].double() - want).abs() <= size * (2 * U[torch.bfloat16] + 4 * tol)).all()


def test_two_handles_on_two_streams_at_once():
    cases = [logprob_case(400, 256, 3000, 1.0, 0.1, seed=s) for s in (41, 42)]
    us = [binding.Update(256, 3000, 400, device=DEV) for _ in cases]
    want = [run_logprob(u, *c[:3], 1.0, c[3]) for u, c in zip(us, cases)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = []
        for u, c, s in zip(us, cases, streams):
            with torch.cuda.stream(s):
                got.append(run_logprob(u, *c[:3], 1.0, c[3]))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(a[k], b[k]) for k in a)


# -------------------------------------------------------------------------------------- expert products

def offsets(counts, start=0):
    return torch.tensor([start] + list(counts), dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)


def expert_reference(kind, off, a, b, E):
    """fp64 values and the sums of absolute products.  fwd: a = x, b = w; dx: a = dy, b = w; dw: a = dy, b = x."""
    o = off.tolist()
    ad, bd = a.double(), b.double()
    if kind == "dw":
        v = torch.zeros(E, a.shape[1], b.shape[1], dtype=torch.float64, device=DEV)
        m = torch.zeros_like(v)
        longest = 1
        for e in range(E):
            r = slice(o[e], o[e + 1])
            longest = max(longest, o[e + 1] - o[e])
            v[e], m[e] = ad[r].t() @ bd[r], ad[r].t().abs() @ bd[r].abs()
        return v, m * sum_error(longest)
    cols = b.shape[1] if kind == "fwd" else b.shape[2]
    v = torch.zeros(a.shape[0], cols, dtype=torch.float64, device=DEV)
    m = torch.zeros_like(v)
    for e in range(E):
        r = slice(o[e], o[e + 1])
        we = bd[e].t() if kind == "fwd" else bd[e]
        v[r], m[r] = ad[r] @ we, ad[r].abs() @ we.abs()
    return v, m * sum_error(a.shape[1])


def check_rounded(got, want, tol):
    r = U[got.dtype]
    assert worst(got, want, tol + r * (want.abs() + tol) + 1e-38) <= 1


CASES = [
    # counts, d_in, d_out, rows in front, rows behind
    ([1], 8, 8, 0, 0), ([0, 3, 0], 64, 72, 0, 0), ([5, 0, 17, 1, 0, 130], 264, 136, 0, 7), ([1] * 8, 256, 512, 0, 0),
    ([128, 64, 16, 15, 33], 128, 256, 3, 5), ([257, 255, 256], 72, 264, 0, 0), ([300, 1, 0, 520], 328, 520, 11, 40),
    ([0, 0, 0], 64, 64, 0, 9), ([700], 520, 264, 1, 0), ([3] * 40, 136, 200, 0, 0)]


@pytest.mark.parametrize("counts,d_in,d_out,before,behind", CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_expert_products_match_the_formula(counts, d_in, d_out, before, behind, dtype):
    E, used = len(counts), sum(counts)
    total = before + used + behind
    g = gen(used + d_in)
    off = offsets(counts, before)
    x, dy, w = normal(g, total, d_in + 8)[:, :d_in], normal(g, total, d_out + 16)[:, :d_out], normal(g, E, d_out, d_in, std=0.1)
    x[:before] = float("nan"); x[before + used:] = float("nan")           # rows that belong to nobody
    dy[:before] = float("inf"); dy[before + used:] = float("nan")
    u = binding.Update(device=DEV)
    mine = slice(before, before + used)
    rest = torch.ones(total, dtype=torch.bool, device=DEV)
    rest[mine] = False
    y = torch.full((total, d_out + 8), 5.0, dtype=dtype, device=DEV)
    assert binding.mars_expert_matmul(u, x, off, w, y[:, :d_out]) == 0
    v, tol = expert_reference("fwd", off, x, w, E)
    check_rounded(y[mine, :d_out], v[mine], tol[mine])
    assert (y[rest] == 5).all() and (y[:, d_out:] == 5).all()
    dx = torch.full((total, d_in + 8), 5.0, dtype=dtype, device=DEV)
    assert binding.mars_expert_matmul_dx(u, dy, off, w, dx[:, :d_in]) == 0
    v, tol = expert_reference("dx", off, dy, w, E)
    check_rounded(dx[mine, :d_in], v[mine], tol[mine])
    assert (dx[rest] == 5).all() and (dx[:, d_in:] == 5).all()
    dw = torch.full((E, d_out, d_in), 5.0, dtype=dtype, device=DEV)
    assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
    v, tol = expert_reference("dw", off, dy, x, E)
    check_rounded(dw, v, tol)
    base = (torch.randn(E, d_out, d_in, generator=g, device=DEV)).to(dtype)
    acc = base.clone()
    assert binding.mars_expert_matmul_dw(u, dy, x, off, acc, accumulate=True) == 0
    want = v + base.double()
    assert worst(acc, want, tol + U[dtype] * (want.abs() + tol) + 2.0 ** -23 * want.abs()) <= 1
    assert u.poll_status() == 0


def test_nothing_crosses_a_group_border():
    """One expert's rows and weights are NaN: only its own outputs are."""
    counts, d_in, d_out = [37, 50, 20, 129], 136, 72
    off, g = offsets(counts), gen(3)
    x, dy, w = normal(g, 236, d_in), normal(g, 236, d_out), normal(g, 4, d_out, d_in)
    u = binding.Update(device=DEV)

    def run(x, dy, w):
        y, dx, dw = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w)
        assert binding.mars_expert_matmul(u, x, off, w, y) == 0
        assert binding.mars_expert_matmul_dx(u, dy, off, w, dx) == 0
        assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
        return y, dx, dw

    clean = run(x, dy, w)
    for e in range(4):
        r = slice(int(off[e]), int(off[e + 1]))
        x2, dy2, w2 = x.clone(), dy.clone(), w.clone()
        x2[r], dy2[r], w2[e] = float("nan"), float("inf"), float("nan")
        got = run(x2, dy2, w2)
        for c, o in zip(clean, got):
            other = torch.ones(o.shape[0], dtype=torch.bool, device=DEV)
            if o.dim() == 3:
                other[e] = False
            else:
                other[r] = False
            assert torch.equal(c[other], o[other])
            assert not torch.isfinite(o[~other]).any()


def test_offsets_outside_the_rows_are_clamped():
    g = gen(2)
    x, dy, w = normal(g, 50, 64), normal(g, 50, 72), normal(g, 5, 72, 64)
    u = binding.Update(device=DEV)
    bad = torch.tensor([-5, 10, 4, 30, 2 ** 31 - 1, 45], dtype=torch.int32, device=DEV)
    good = torch.tensor([0, 10, 10, 30, 50, 50], dtype=torch.int32, device=DEV)
    res = []
    for off in (bad, good):
        y, dx, dw = torch.zeros_like(dy), torch.zeros_like(x), torch.empty_like(w)
        assert binding.mars_expert_matmul(u, x, off, w, y) == 0
        assert binding.mars_expert_matmul_dx(u, dy, off, w, dx) == 0
        assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
        res.append((y, dx, dw))
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_many_experts_and_no_rows():
    u = binding.Update(device=DEV)
    g = gen(9)
    E = 1024
    counts = [(i * 7) % 4 for i in range(E)]
    off, used = offsets(counts), sum(counts)
    x, dy, w = normal(g, used, 64), normal(g, used, 40), normal(g, E, 40, 64)
    y = torch.empty_like(dy)
    assert binding.mars_expert_matmul(u, x, off, w, y) == 0
    check_rounded(y, *expert_reference("fwd", off, x, w, E))
    dw = torch.full_like(w, 2.0)
    assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
    check_rounded(dw, *expert_reference("dw", off, dy, x, E))
    none = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    for rows in (0, 5):
        dw.fill_(2.0)
        assert binding.mars_expert_matmul_dw(u, dy[:rows], x[:rows], none, dw, accumulate=True) == 0
        assert (dw == 2).all()
        assert binding.mars_expert_matmul_dw(u, dy[:rows], x[:rows], none, dw) == 0
        assert (dw == 0).all()
        y2 = torch.full((rows, 40), 3.0, device=DEV)
        assert binding.mars_expert_matmul(u, x[:rows], none, w, y2) == 0 and (y2 == 3).all()


def test_expert_stack_beyond_32_bit_offsets():
    """2.7e9 weights: the last expert's rows, and a border between experts behind 2^31 elements."""
    E, d = 40, 8192
    counts = [0] * E
    counts[0], counts[31], counts[32], counts[E - 1] = 2, 20, 5, 17
    off, g = offsets(counts), gen(33)
    n = sum(counts)
    w = torch.empty(E, d, d, dtype=torch.bfloat16, device=DEV)
    w.normal_(std=0.02, generator=g)
    x, dy = normal(g, n, d), normal(g, n, d)
    u = binding.Update(device=DEV)
    y, dx = torch.empty_like(dy), torch.empty_like(x)
    assert binding.mars_expert_matmul(u, x, off, w, y) == 0
    assert binding.mars_expert_matmul_dx(u, dy, off, w, dx) == 0
    dw = torch.full_like(w, 9.0)
    assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
    o = off.tolist()
    for e in (0, 31, 32, E - 1):
        r = slice(o[e], o[e + 1])
        we, xe, dye = w[e].double(), x[r].double(), dy[r].double()
        check_rounded(y[r], xe @ we.t(), sum_error(d) * (xe.abs() @ we.abs().t()))
        check_rounded(dx[r], dye @ we, sum_error(d) * (dye.abs() @ we.abs()))
        check_rounded(dw[e], dye.t() @ xe, sum_error(20) * (dye.abs().t() @ xe.abs()))
    assert (dw[1:31] == 0).all() and (dw[33:E - 1] == 0).all()


def in_parts(n):
    """Relative to the sum of absolute products: at most 4096 indexes in one tensor-core sum, the parts added in fp32."""
    return sum_error(min(n, 4096)) + -(-n // 4096) * 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_groups_do_not_lose_what_each_step_drops(dtype):
    """Products of one sign, where the low bits that the tensor cores drop add up: the bound does not grow with the group."""
    counts, d_in, d_out = [30000, 4096, 0, 4097, 8192, 12345, 63, 16384], 136, 328
    off, g, u = offsets(counts), gen(61), binding.Update(device=DEV)
    n, E = sum(counts), len(counts)
    x, dy = normal(g, n, d_in).abs(), normal(g, n, d_out).abs()
    base = torch.rand(E, d_out, d_in, generator=g, device=DEV).to(dtype)
    dw, acc = torch.empty(E, d_out, d_in, dtype=dtype, device=DEV), base.clone()
    assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
    assert binding.mars_expert_matmul_dw(u, dy, x, off, acc, accumulate=True) == 0
    o = off.tolist()
    for e in range(E):
        want = dy[o[e]:o[e + 1]].double().t() @ x[o[e]:o[e + 1]].double()
        tol = want * in_parts(counts[e])
        check_rounded(dw[e], want, tol)
        check_rounded(acc[e], want + base[e].double(), tol + 2.0 ** -23 * want)
    assert u.poll_status() == 0


def test_wide_experts_do_not_lose_what_each_step_drops():
    counts, d = [5, 300, 0, 41], 20008
    off, g, u = offsets(counts), gen(62), binding.Update(device=DEV)
    n = sum(counts)
    x, w = normal(g, n, d).abs(), normal(g, 4, 264, d).abs()
    y = torch.empty(n, 264, device=DEV)
    assert binding.mars_expert_matmul(u, x, off, w, y) == 0
    wt = w.transpose(1, 2).contiguous()
    dx = torch.empty(n, 264, device=DEV)
    assert binding.mars_expert_matmul_dx(u, x, off, wt, dx) == 0          # the same sums, w the other way round
    o = off.tolist()
    for e in range(4):
        r = slice(o[e], o[e + 1])
        want = x[r].double() @ w[e].double().t()
        for got in (y[r], dx[r]):
            check_rounded(got, want, want * in_parts(d))


def test_lm_head_gradient_of_many_rows_does_not_lose_what_each_step_drops():
    """Two entries of equal logits: p is 1/2 and d exact in bf16, so that nothing but the sum over the rows can be off."""
    n, H = 30011, 72
    g = gen(63)
    h = normal(g, n, H).abs()
    w = normal(g, 1, H).expand(2, H).contiguous()
    targets = torch.zeros(n, dtype=torch.int32, device=DEV)
    targets[::1000] = -1
    u = binding.Update(H, 2, n, device=DEV)
    got = run_logprob(u, h, w, targets, 1.0, torch.ones(n, device=DEV), dtype=torch.float32)
    half = 0.5 * torch.where((targets >= 0)[:, None], h.double(), 0.0).sum(0)
    for row, want in ((0, half), (1, -half)):
        check_rounded(got["d_w"][row], want, half * in_parts(n))


def test_a_group_of_four_hundred_million_rows():
    """Six million stages on one pair of CTAs: the work of seconds must not look like a wait that gave up."""
    n, d = 400_000_000, 8
    u, g = binding.Update(device=DEV), gen(64)
    x, dy = (torch.empty(n, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    x.uniform_(0.5, 1.0, generator=g)
    dy.uniform_(0.5, 1.0, generator=g)
    dw = torch.empty(2, d, d, device=DEV)
    off = torch.tensor([0, n - 5, n], dtype=torch.int32, device=DEV)
    assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
    assert u.poll_status() == 0
    want = torch.zeros(d, d, dtype=torch.float64, device=DEV)
    for a in range(0, n - 5, 10_000_000):
        b = min(a + 10_000_000, n - 5)
        want += dy[a:b].double().t() @ x[a:b].double()
    check_rounded(dw[0], want, want * in_parts(n))
    check_rounded(dw[1], dy[n - 5:].double().t() @ x[n - 5:].double(), 5 * sum_error(5) * torch.ones(d, d, device=DEV))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_groups_of_more_rows_than_a_block_of_tiles(dtype):
    """Groups whose rows exceed what is kept in L2 while the weights pass: at a width of 16384 that is 1024 rows, at 4104
    3840, with the last block full, ragged, of one row."""
    for counts, d, o in (([2500, 0, 1024, 1025, 300], 16384, 520), ([9000, 3840, 3841], 4104, 264)):
        off, g, u = offsets(counts, 3), gen(92), binding.Update(device=DEV)
        n, E = sum(counts) + 3, len(counts)
        x, w = normal(g, n, d), normal(g, E, o, d, std=0.1)
        y = torch.full((n, o), 5.0, dtype=dtype, device=DEV)
        assert binding.mars_expert_matmul(u, x, off, w, y) == 0
        wt = w.transpose(1, 2).contiguous()
        dx = torch.full((n, o), 5.0, dtype=dtype, device=DEV)
        assert binding.mars_expert_matmul_dx(u, x, off, wt, dx) == 0       # the same sums, w the other way round
        v, tol = expert_reference("fwd", off, x, w, E)
        for got in (y, dx):
            check_rounded(got[3:], v[3:], tol[3:])
            assert (got[:3] == 5).all()
        assert u.poll_status() == 0


def test_expert_gradients_against_differences():
    """L = sum_r <c_r, w_e x_r> in fp64 along random directions of x and w."""
    counts, d_in, d_out = [9, 0, 40, 131], 72, 88
    off, g = offsets(counts), gen(6)
    n, E = sum(counts), len(counts)
    x, c, w = normal(g, n, d_in), normal(g, n, d_out), normal(g, E, d_out, d_in)
    u = binding.Update(device=DEV)
    dx, dw = torch.empty(n, d_in, device=DEV), torch.empty(E, d_out, d_in, device=DEV)
    assert binding.mars_expert_matmul_dx(u, c, off, w, dx) == 0
    assert binding.mars_expert_matmul_dw(u, c, x, off, dw) == 0
    e_of = torch.repeat_interleave(torch.arange(E, device=DEV), torch.tensor(counts, device=DEV))

    def loss(xd, wd):
        return float((c.double() * torch.einsum("nk,nok->no", xd, wd[e_of])).sum())

    for _ in range(4):
        for grad, at in ((dx, 0), (dw, 1)):
            base = [x.double(), w.double()]
            v = torch.randn(base[at].shape, generator=g, device=DEV, dtype=torch.float64)
            up, dn = list(base), list(base)
            up[at], dn[at] = base[at] + 0.5 * v, base[at] - 0.5 * v       # the loss is linear in each
            diff = loss(*up) - loss(*dn)
            size = float((grad.double().abs() * v.abs()).sum())
            assert abs(float((grad.double() * v).sum()) - diff) <= 1e-5 * size


def test_expert_products_in_a_graph_follow_new_offsets():
    g = gen(11)
    x, dy, w = normal(g, 400, 128), normal(g, 400, 136), normal(g, 6, 136, 128)
    off = offsets([100, 50, 0, 20, 30, 100])
    u = binding.Update(device=DEV)
    y, dx, dw = torch.zeros_like(dy), torch.zeros_like(x), torch.zeros_like(w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert binding.mars_expert_matmul(u, x, off, w, y) == 0
        assert binding.mars_expert_matmul_dx(u, dy, off, w, dx) == 0
        assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
    for counts in ([100, 50, 0, 20, 30, 100], [1, 2, 3, 4, 380, 10]):
        off.copy_(offsets(counts))
        n = sum(counts)
        graph.replay()
        torch.cuda.synchronize()
        v, tol = expert_reference("fwd", off, x, w, 6)
        check_rounded(y[:n], v[:n], tol[:n])
        v, tol = expert_reference("dx", off, dy, w, 6)
        check_rounded(dx[:n], v[:n], tol[:n])
        check_rounded(dw, *expert_reference("dw", off, dy, x, 6))


def test_expert_refusals():
    u = binding.Update(device=DEV)
    x, w, y = (torch.zeros(*s, dtype=torch.bfloat16, device=DEV) for s in ((6, 64), (2, 64, 64), (6, 64)))
    off = offsets([3, 3])
    assert binding.mars_expert_matmul(u, x, off, w, x) == 1
    assert binding.mars_expert_matmul_dx(u, x, off, w, x) == 1
    assert binding.mars_expert_matmul_dw(u, x, x, off, w.view(2, 64, 64)) == 0
    buf = torch.zeros(4 * 64 * 64, dtype=torch.bfloat16, device=DEV)
    assert binding.mars_expert_matmul_dw(u, buf[:6 * 64].view(6, 64), x, off, buf[64:64 + 2 * 64 * 64].view(2, 64, 64)) == 1
    w9 = torch.zeros(2, 64, 12, dtype=torch.bfloat16, device=DEV)
    assert binding.mars_expert_matmul(u, torch.zeros(6, 12, dtype=torch.bfloat16, device=DEV), off, w9, y) == 1
    odd = torch.zeros(6, 66, dtype=torch.bfloat16, device=DEV)[:, :64]
    assert binding.mars_expert_matmul(u, odd, off, w, y) == 1
    many = torch.zeros(1025, 8, 8, dtype=torch.bfloat16, device=DEV)
    assert binding.mars_expert_matmul(u, x[:, :8], torch.zeros(1026, dtype=torch.int32, device=DEV), many, y[:, :8]) == 1
    assert u.poll_status() == 0


def test_more_rows_than_an_index_holds_are_refused():
    """The C entry itself: nothing is launched, so the row count need not be backed by memory."""
    u = binding.Update(device=DEV)
    x, w = torch.zeros(6, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 64, 64, dtype=torch.bfloat16, device=DEV)
    y, off = torch.full_like(x, 3.0), offsets([3, 3])
    call = binding.lib().mars_expert_matmul
    for rows in (-1, (1 << 30) + 1, (1 << 31) - 1):
        assert call(u.handle, u._stream(None), 2, rows, 64, 64, x.data_ptr(), 64, off.data_ptr(), w.data_ptr(), y.data_ptr(), 64, 1) == 1
    torch.cuda.synchronize()
    assert (y == 3).all()


def test_inputs_and_outputs_side_by_side_in_one_buffer():
    """Column ranges of one [rows][...] buffer do not overlap; ranges that share a column, or reach into the next row, do."""
    counts, d, o = [40, 0, 33], 64, 72
    off, g, u, n = offsets(counts), gen(81), binding.Update(device=DEV), 73
    w = normal(g, 3, o, d)
    buf = normal(g, n + 1, 160)
    x, dy = buf[:n, :d].clone(), normal(g, n, o)
    y = torch.empty(n, o, dtype=torch.bfloat16, device=DEV)
    dx = torch.empty_like(x)
    assert binding.mars_expert_matmul(u, x, off, w, y) == 0 and binding.mars_expert_matmul_dx(u, dy, off, w, dx) == 0
    rest = buf.clone()
    assert binding.mars_expert_matmul(u, buf[:n, :d], off, w, buf[:n, d:d + o]) == 0
    assert torch.equal(buf[:n, d:d + o], y)
    rest[:n, d:d + o] = y
    assert torch.equal(buf, rest)
    buf[:n, :o] = dy                                                # the output in front or behind, and of four bytes
    assert binding.mars_expert_matmul_dx(u, buf[:n, :o], off, w, buf[:n, 96:96 + d]) == 0
    assert torch.equal(buf[:n, 96:96 + d], dx) and torch.equal(buf[:n, :o], dy)
    buf[:n, 80:80 + o] = dy
    assert binding.mars_expert_matmul_dx(u, buf[:n, 80:80 + o], off, w, buf[:n, 8:8 + d]) == 0
    assert torch.equal(buf[:n, 8:8 + d], dx)
    wide = torch.zeros(n, 256, device=DEV)                          # fp32 rows of 1024 bytes; x in the first 128 of them
    half = wide.view(torch.bfloat16)
    half[:, :d] = x
    assert binding.mars_expert_matmul(u, half[:, :d], off, w, wide[:, 64:64 + o]) == 0
    assert torch.equal(wide[:, 64:64 + o].bfloat16(), y) and torch.equal(half[:, :d], x)
    before = buf.clone()
    for a, b in ((0, 56), (56, 0), (8, 64)):                       # shared columns
        assert binding.mars_expert_matmul(u, buf[:n, a:a + d], off, w, buf[:n, b:b + o]) == 1
    late = buf.view(-1)[120:120 + n * 160].view(n, 160)             # begins in a row's columns 120 .. and ends in the next row's
    assert binding.mars_expert_matmul(u, buf[:n, :d], off, w, late[:, :o]) == 1
    assert binding.mars_expert_matmul(u, late[:, :d], off, w, buf[:n, :o]) == 1
    narrow = buf.view(-1)[:n * 80].view(n, 80)                      # other row strides
    assert binding.mars_expert_matmul(u, narrow[:, :d], off, w, buf[:n, d:d + o]) == 1
    torch.cuda.synchronize()
    assert torch.equal(buf, before)


def test_hidden_and_its_gradient_side_by_side_in_one_buffer():
    h, lm, targets, d = logprob_case(90, 64, 500, 1.0, 0.2, seed=82)
    u = binding.Update(64, 500, 90, device=DEV)
    want = run_logprob(u, h, lm, targets, 1.0, d)
    buf = torch.full((90, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    buf[:, :64] = h
    d_w = torch.empty_like(lm)
    assert binding.mars_logprob_grad(u, buf[:, :64], lm, targets, 1.0, want["lse"], d, buf[:, 64:], d_w) == 0
    assert torch.equal(buf[:, 64:], want["d_h"]) and torch.equal(buf[:, :64], h) and torch.equal(d_w, want["d_w"])
    assert binding.mars_logprob_grad(u, buf[:, :64], lm, targets, 1.0, want["lse"], d, buf[:, 56:120], d_w) == 1


def test_wider_experts_than_an_index_holds_are_refused():
    """The C entries themselves: nothing is launched, so the sizes need not be backed by memory."""
    u = binding.Update(device=DEV)
    x, w, y, off = torch.zeros(64, device=DEV), torch.zeros(64, device=DEV), torch.full((64,), 3.0, device=DEV), offsets([1])
    L, p = binding.lib(), [t.data_ptr() for t in (x, w, y)]
    top = (1 << 31) - 8
    for d_in, d_out in ((8, top), (top, 8), ((1 << 30) + 8, 8), (8, (1 << 30) + 8)):
        assert L.mars_expert_matmul(u.handle, None, 1, 1, d_in, d_out, p[0], d_in, off.data_ptr(), p[1], p[2], d_out, 1) == 1
        assert L.mars_expert_matmul_dx(u.handle, None, 1, 1, d_in, d_out, p[0], d_out, off.data_ptr(), p[1], p[2], d_in, 1) == 1
        assert L.mars_expert_matmul_dw(u.handle, None, 1, 1, d_in, d_out, p[0], d_out, p[1], d_in, off.data_ptr(), p[2], 1, 0) == 1
    torch.cuda.synchronize()
    assert (y == 3).all()


# -------------------------------------------------------------------------------------- gradient lists

def grad_tensors(sizes, types, seed, aligned=True, std=1.0):
    """Views into one flat buffer per type, at odd places unless aligned."""
    g = gen(seed)
    pad = 64 if aligned else 1
    flat = {t: torch.zeros(sum(-(-n // pad) * pad for n, q in zip(sizes, types) if q == t) + 65, dtype=t, device=DEV) for t in set(types)}
    at, out = {t: (0 if aligned else 1) for t in flat}, []
    for n, t in zip(sizes, types):
        v = flat[t][at[t]:at[t] + n]
        v.copy_(torch.randn(n, generator=g, device=DEV) * std)
        at[t] += -(-n // pad) * pad
        out.append(v)
    return flat, out


def check_clip(before, after, norm, max_norm):
    want = math.sqrt(math.fsum(float(t.double().square().sum()) for t in before))
    # fp32 sums over at most 65 squares of a thread (2^-24 each), fp64 beyond; one rounding of the norm and of the scale
    rel = 65 * 2.0 ** -24
    assert abs(float(norm) - want) <= (rel + 2.0 ** -24) * want
    scale = min(1.0, max_norm / (want + 1e-6))
    for b, a in zip(before, after):
        v = b.double() * scale
        tol = v.abs() * (U[b.dtype] + rel + 2.0 ** -23) + (2.0 ** -25 if b.dtype == torch.float16 else 0)     # fp16: half its smallest step
        assert worst(a, v, tol) <= 1


F32, BF, HF = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("sizes,types", [
    ([1], [F32]), ([1], [BF]), ([7, 1, 0, 3], [HF, BF, F32, F32]), ([0, 0], [F32, BF]), ([100, 5, 33], [F32] * 3),
    ([16384, 16383, 16385, 8191, 8193, 32769], [BF, BF, HF, F32, F32, BF]), ([1] * 300, [BF, F32, HF] * 100),
    ([1000003, 17, 250000], [BF, HF, F32]), ([3_000_000, 2_000_001], [F32, BF])])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("ratio", [0.3, 2.0])
def test_clip_matches_the_formula(sizes, types, aligned, ratio):
    flat, grads = grad_tensors(sizes, types, seed=len(sizes), aligned=aligned)
    before = [t.clone() for t in grads]
    all_before = {t: v.clone() for t, v in flat.items()}
    max_norm = ratio * math.sqrt(max(1, sum(sizes)))
    norm = torch.full((1,), -1.0, device=DEV)
    # into other tensors, at other places of theirs
    out_flat, outs = grad_tensors(sizes, types, seed=99, aligned=not aligned)
    lst = binding.GradList(grads, outs)
    assert binding.mars_grads_norm(lst, norm) == 0
    check_clip(before, before, norm, math.inf)
    assert binding.mars_grads_clip(lst, max_norm, norm) == 0
    check_clip(before, outs, norm, max_norm)
    for t, v in flat.items():
        assert torch.equal(v, all_before[t])
    # in place, neighbours untouched
    lst = binding.GradList(grads)
    assert binding.mars_grads_clip(lst, max_norm, norm) == 0
    check_clip(before, grads, norm, max_norm)
    for t, v in flat.items():
        gaps = torch.ones_like(v, dtype=torch.bool)
        for q in grads:
            if q.dtype == t:
                a = (q.data_ptr() - v.data_ptr()) // q.element_size()
                gaps[a:a + q.numel()] = False
        assert torch.equal(v[gaps], all_before[t][gaps])


@pytest.mark.parametrize("value", [1e30, 1e-30, 3e-39])
def test_norms_whose_squares_leave_the_range_of_fp32(value):
    t = torch.full((5000,), value, device=DEV)
    b = torch.full((77,), value, device=DEV).bfloat16()
    norm = torch.empty(1, device=DEV)
    assert binding.mars_grads_norm(binding.GradList([t, b]), norm) == 0
    want = math.sqrt(float(t.double().square().sum()) + float(b.double().square().sum()))
    assert abs(float(norm) - want) <= 1e-5 * want


@pytest.mark.parametrize("value,max_norm,count", [(3e38, 1.0, 100_003), (3e38, 1e-3, 777), (1e10, 1e-30, 100), (2e38, 1e-20, 50), (3.0, 1e-37, 9),
                                                  (1e20, 3e-18, 300)])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("odd", [0, 1])
def test_factors_below_the_normal_numbers_of_fp32(value, max_norm, count, dtype, odd):
    """max_norm / norm from 1e-37 down to 1e-60: results that fp32 holds are right all the same."""
    t = (torch.rand(count + 1, generator=gen(3), device=DEV) * 0.5 + 0.5).mul_(value).to(dtype)[odd:count + odd]
    o, norm = torch.full((count,), 7.0, dtype=dtype, device=DEV), torch.empty(1, device=DEV)
    want_norm = math.sqrt(float((t.double() / value).square().sum())) * value
    scale = max_norm / (want_norm + 1e-6)
    assert binding.mars_grads_clip(binding.GradList([t], [o]), max_norm, norm) == 0
    want = t.double() * scale
    tol = want.abs() * (U[dtype] + 66 * 2.0 ** -24 + 2.0 ** -23) + (2.0 ** -150 if dtype == F32 else 2.0 ** -134 + 2.0 ** -150)
    assert worst(o, want, tol) <= 1
    assert binding.mars_grads_clip(binding.GradList([t]), max_norm, norm) == 0            # in place
    assert torch.equal(t, o)


def test_infinities_and_nan():
    norm = torch.empty(1, device=DEV)
    t = torch.ones(1000, device=DEV)
    t[500] = float("inf")
    o = torch.empty_like(t)
    assert binding.mars_grads_clip(binding.GradList([t], [o]), 1.0, norm) == 0
    assert math.isinf(float(norm)) and float(o[0]) == 0 and math.isnan(float(o[500]))
    t[500] = float("nan")
    assert binding.mars_grads_clip(binding.GradList([t], [o]), 1.0, norm) == 0
    assert math.isnan(float(norm)) and torch.isnan(o).all()
    z = torch.zeros(10, device=DEV)
    assert binding.mars_grads_clip(binding.GradList([z]), 0.0, norm) == 0
    assert float(norm) == 0 and (z == 0).all()


def test_clip_is_the_same_every_time_and_in_a_graph():
    flat, grads = grad_tensors([500001, 77, 123456], [BF, F32, HF], seed=4, aligned=False)
    outs = [torch.zeros_like(t) for t in grads]
    lst = binding.GradList(grads, outs)
    norm = torch.zeros(1, device=DEV)
    assert binding.mars_grads_clip(lst, 10.0, norm) == 0
    first = [norm.clone()] + [t.clone() for t in outs]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert binding.mars_grads_clip(lst, 10.0, norm) == 0
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, [norm] + outs))
    grads[0].mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    check_clip(grads, outs, norm, 10.0)


def test_a_tensor_beyond_32_bit_offsets():
    n = 2 ** 32 + 12345
    t = torch.full((n,), 0.5, dtype=torch.bfloat16, device=DEV)
    t[-1], t[2 ** 31 + 7] = 300.0, -200.0
    norm = torch.empty(1, device=DEV)
    lst = binding.GradList([t[1:]])
    assert binding.mars_grads_clip(lst, 100.0, norm) == 0
    want = math.sqrt(0.25 * (n - 3) + 300.0 ** 2 + 200.0 ** 2)
    assert abs(float(norm) - want) <= 66 * 2.0 ** -24 * want
    s = 100.0 / want
    for i, v in ((0, 0.5), (1, 0.5 * s), (2 ** 31 + 7, -200.0 * s), (2 ** 32, 0.5 * s), (n - 2, 0.5 * s), (n - 1, 300.0 * s)):
        assert abs(float(t[i]) - v) <= abs(v) * (U[BF] + 1e-5), i
    assert float(t[2 ** 32:].float().sum()) == pytest.approx(float(t[2].float()) * (12345 - 1) + float(t[-1]), rel=1e-5)


def test_grad_list_refusals():
    t = torch.ones(64, device=DEV)
    norm = torch.empty(1, device=DEV)
    lst = binding.GradList([t])
    assert binding.mars_grads_clip(lst, -1.0, norm) == 1 and binding.mars_grads_clip(lst, float("nan"), norm) == 1
    with pytest.raises(binding.MarsError):
        binding.GradList([t, t])                      # scaled twice
    with pytest.raises(binding.MarsError):
        binding.GradList([t[:32], t[16:]])
    twice = binding.GradList([t, t], [torch.empty_like(t), torch.empty_like(t)])      # counted twice, written apart
    assert binding.mars_grads_norm(twice, norm) == 0 and abs(float(norm) - math.sqrt(128)) < 1e-4
    with pytest.raises(ValueError):
        binding.mars_grads_norm(lst, torch.empty(2, device=DEV))


# ------------------------------------------------------------------------- handles and streams

def test_a_new_handle_is_ready_for_any_stream():
    """A side stream does not wait for the legacy stream, which is busy while the handles are made."""
    h, w, targets, _ = logprob_case(8, 64, 100, 1.0, seed=5)
    targets[3] = 100                                                    # beyond the vocabulary
    lp, lse, norm = torch.empty(8, device=DEV), torch.empty(8, device=DEV), torch.empty(1, device=DEV)
    t = torch.ones(64, device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(400_000_000)                                      # about 0.2 s on the legacy stream
    with torch.cuda.stream(side):
        u, lst = binding.Update(64, 100, 8, device=DEV), binding.GradList([t])
        assert binding.mars_logprob(u, h, w, targets, 1.0, lp, lse) == 0
        assert binding.mars_grads_norm(lst, norm) == 0
    side.synchronize()
    assert u.poll_status() == 7 and u.poll_status() == 0
    assert float(norm) == 8.0 and float(lp[3]) == 0.0


def test_the_status_of_a_replay_is_waited_for():
    """The graph is replayed on another stream than it was captured on, behind other work, and polled at once."""
    h, w, targets, _ = logprob_case(8, 64, 100, 1.0, seed=5)
    targets[3] = 100
    u, (lp, lse) = binding.Update(64, 100, 8, device=DEV), torch.empty(2, 8, device=DEV)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        assert binding.mars_logprob(u, h, w, targets, 1.0, lp, lse) == 0
    assert u.poll_status() == 0                                         # captured, not run
    for _ in range(2):
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)
            graph.replay()
        assert u.poll_status() == 7 and u.poll_status() == 0
    # the handle outlives the stream of its last call
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert binding.mars_logprob(u, h, w, targets, 1.0, lp, lse) == 0
    del s
    assert u.poll_status() == 7


def test_a_workspace_is_not_handed_on_while_a_side_stream_uses_it():
    t, norm = torch.ones(64, device=DEV), torch.empty(1, device=DEV)
    lst = binding.GradList([t])
    at, nbytes = lst.workspace.data_ptr(), lst.workspace.numel()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
        assert binding.mars_grads_clip(lst, 1.0, norm) == 0
    lst.close()
    del lst
    others = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(4)]       # never written to
    assert not side.query() and all(o.data_ptr() != at for o in others)
    side.synchronize()
    assert float(norm) == 8.0 and abs(float(t[0]) - 0.125) < 1e-6


def test_every_contraction_again_and_again():
    """Many ring rounds, tiles and launches of every kind of epilogue back to back: the same bits each time, no wait that
    gives up."""
    h, w, targets, d = logprob_case(640, 512, 5000, 1.0, 0.1, seed=51)
    u, few = binding.Update(512, 5000, 640, device=DEV), slice(0, 90)
    first, short = run_logprob(u, h, w, targets, 1.0, d), run_logprob(u, h[few], w, targets[few], 1.0, d[few])
    off, g = offsets([300, 0, 77, 1, 512, 90]), gen(52)
    x, dy, ew = normal(g, 980, 512), normal(g, 980, 768), normal(g, 6, 768, 512)

    def products():
        y, dx, dw = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(ew)
        assert binding.mars_expert_matmul(u, x, off, ew, y) == 0
        assert binding.mars_expert_matmul_dx(u, dy, off, ew, dx) == 0
        assert binding.mars_expert_matmul_dw(u, dy, x, off, dw) == 0
        return dict(y=y, dx=dx, dw=dw)

    want = products()
    for _ in range(60):
        for a, b in ((first, run_logprob(u, h, w, targets, 1.0, d)), (want, products()),
                     (short, run_logprob(u, h[few], w, targets[few], 1.0, d[few]))):
            assert all(torch.equal(a[k], b[k]) for k in a)
    assert u.poll_status() == 0


# ----------------------------------------------------------------------------------- as they are used

def test_an_update_of_the_last_expert_layer_and_the_lm_head():
    """Expert products -> hidden states -> log-probs -> their gradient -> expert gradients -> clipping, every
    intermediate taken as the kernels rounded it, each stage against fp64 on its own inputs."""
    g = gen(21)
    counts, d_in, H, V, T = [40, 0, 75, 13], 136, 128, 1100, 0.85
    off, n, E = offsets(counts), 128, 4
    x, w, lm = normal(g, n, d_in), normal(g, E, H, d_in, std=0.1), normal(g, V, H, std=0.1)
    targets = torch.randint(V, (n,), generator=g, device=DEV, dtype=torch.int32)
    targets[::5] = -1
    weight = torch.randn(n, generator=g, device=DEV) / n
    u = binding.Update(H, V, n, device=DEV)
    y = torch.empty(n, H, dtype=torch.bfloat16, device=DEV)
    assert binding.mars_expert_matmul(u, x, off, w, y) == 0
    check_rounded(y, *expert_reference("fwd", off, x, w, E))
    got = run_logprob(u, y, lm, targets, T, weight)
    check_logprob(got, logprob_reference(y, lm, targets, T, weight))
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    assert binding.mars_expert_matmul_dx(u, got["d_h"], off, w, dx) == 0
    assert binding.mars_expert_matmul_dw(u, got["d_h"], x, off, dw) == 0
    check_rounded(dx, *expert_reference("dx", off, got["d_h"], w, E))
    check_rounded(dw, *expert_reference("dw", off, got["d_h"], x, E))
    before = [got["d_w"].clone(), dw.clone()]
    norm = torch.empty(1, device=DEV)
    lst = binding.GradList([got["d_w"], dw])
    assert binding.mars_grads_clip(lst, 1e-3, norm) == 0
    check_clip(before, [got["d_w"], dw], norm, 1e-3)
    assert float(norm) > 1e-3 and u.poll_status() == 0
