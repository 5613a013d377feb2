"""Operators of a training pass on the GPU against plain 64-bit forms: norms, rotation, router and policy loss with their
gradients.

Tolerances are bounds from the arithmetic, evaluated on each test's own inputs.  u(t) = half a step of type t (bf16 2^-8, fp16
2^-11, fp32 2^-24, relative to the value), V = u(fp32).  A sum of n fp32 terms that c of them meet in a chain is off by at most
c V times the sum of the absolute terms; chains here are 32 values of a thread and the 5 + 16 joins of its block at most.
"""
import math
from decimal import localcontext

import pytest
import torch

from helpers import TWO_PI, exact_frequencies
from paper_2511_11373_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
F, B, H = torch.float32, torch.bfloat16, torch.float16
U = {B: 2.0 ** -8, H: 2.0 ** -11, F: 2.0 ** -24}
SMALLEST = {B: 2.0 ** -134, H: 2.0 ** -25, F: 2.0 ** -150}       # half a step below the normal numbers
V = 2.0 ** -24
RMS, LAYER = binding.MARS_NORM_RMS, binding.MARS_NORM_LAYER


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape, std=1.0, mean=0.0, dtype=F):
    return (torch.randn(*shape, generator=g, device=DEV) * std + mean).to(dtype)


def worst(got, want, tol):
    """Largest error in units of its tolerance (NaN counts as infinite)."""
    e = (got.double() - want).abs() / tol.clamp_min(1e-300)
    e = torch.where(got.double() == want, torch.zeros_like(e), e)
    return float(torch.nan_to_num(e, nan=math.inf).max()) if e.numel() else 0.0


def rounded(t, want, tol):
    return tol + U[t] * (want.abs() + tol) + SMALLEST[t]


def inside(shape, dtype, g, pad, std=1.0, mean=0.0):
    """A tensor [n, ...] inside rows that are `pad` elements longer; what is beside it is NaN."""
    n, cols = shape[0], math.prod(shape[1:])
    buf = torch.full((n, cols + pad), math.nan, device=DEV, dtype=dtype)
    buf[:, :cols] = normal(g, n, cols, std=std, mean=mean, dtype=dtype)
    return buf, buf[:, :cols].unflatten(1, shape[1:]) if len(shape) == 3 else buf[:, :cols]


# ------------------------------------------------------------------------------------------------- norms

EPS = 1e-6


def norm_reference(kind, x, w, b, add=None):
    s = x if add is None else (x.double() + add.double()).to(F).to(x.dtype)      # fp32, then the type of x
    d = s.double()
    mean = d.mean(-1, keepdim=True) if kind == LAYER else torch.zeros_like(d[..., :1])
    u = d - mean
    r = (u.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = u * r * w.double() + (b.double() if b is not None else 0)
    # mean: a chain of 64 additions and a product; the squares' sum the same, half of it in the root, + root and quotient
    off = 64 * V * d.abs().mean(-1, keepdim=True) if kind == LAYER else torch.zeros_like(mean)
    tol = (r * w.double()).abs() * (off * 2 + 64 * V * u.abs()) + V * (y.abs() + (b.double().abs() if b is not None else 0))
    return dict(s=s, y=y, tol=tol, rstd=r[..., 0], mean=mean[..., 0], tol_mean=off[..., 0] + 1e-300,
                tol_rstd=(r * (64 * V + off * r))[..., 0])


def norm_grad_reference(kind, dy, x, w, mean, rstd, d_sum=None):
    """From the formulas, with the statistics as given; tolerances beside."""
    d, r, W = dy.double(), rstd.double()[..., None], x.shape[-1]
    n = (x.double() - (mean.double()[..., None] if kind == LAYER else 0)) * r
    g = d * w.double()
    c0 = (g * n).mean(-1, keepdim=True)
    c1 = g.mean(-1, keepdim=True) if kind == LAYER else torch.zeros_like(c0)
    dx = r * (g - n * c0 - c1)
    e0, e1 = 64 * V * (g * n).abs().mean(-1, keepdim=True), (64 * V * g.abs().mean(-1, keepdim=True) if kind == LAYER else 0 * c0)
    tol = r * (8 * V * (g.abs() + c1.abs() + (n * c0).abs()) + n.abs() * e0 + e1)
    if d_sum is not None:
        dx = dx + d_sum.double()
        tol = tol + V * (dx.abs() + d_sum.double().abs())
    flat = lambda t: t.reshape(-1, W)
    rows = flat(d).shape[0]
    # rows of a thread (the grid has 148 blocks at least), threads of a block that share a column (256 at most), product and n
    chain = (rows / 148 + 262) * V
    return dict(dx=dx, tol_dx=tol, dw=flat(d * n).sum(0), db=flat(d).sum(0), tol_dw=chain * flat((d * n).abs()).sum(0),
                tol_db=chain * flat(d.abs()).sum(0))


def norm_case(kind, shape, xt, yt, wt, pad=0, seed=0, add=False, bias=False):
    g = gen(seed)
    W = shape[-1]
    c = dict(kind=kind, x=inside(shape, xt, g, pad, 1.5, 0.3)[1], w=normal(g, W, std=0.2, mean=1.0, dtype=wt),
             b=normal(g, W, std=0.3, dtype=wt) if bias else None, dy=inside(shape, yt, g, pad, 0.5)[1],
             add=inside(shape, yt, g, pad, 0.7)[1] if add else None, d_sum=inside(shape, xt, g, pad, 0.4)[1] if add else None)
    return c


def out_like(shape, dtype, pad):
    buf = torch.full((shape[0], math.prod(shape[1:]) + pad), 77.0, device=DEV, dtype=dtype)
    view = buf[:, :math.prod(shape[1:])]
    return buf, view.unflatten(1, shape[1:]) if len(shape) == 3 else view


def run_norm(train, c, yt, pad=0, stats=True, stream=None):
    x, kind = c["x"], c["kind"]
    rows = x.shape[:-1]
    buf, y = out_like(x.shape, yt, pad)
    got = dict(y=y, buf=buf)
    if stats:
        got["rstd"] = torch.full(rows, 77.0, device=DEV)
        got["mean"] = torch.full(rows, 77.0, device=DEV) if kind == LAYER else None
    if c["add"] is not None:
        got["s_buf"], got["s"] = out_like(x.shape, x.dtype, pad)
    assert binding.mars_norm(train, kind, x, c["w"], EPS, y, rstd=got.get("rstd"), mean=got.get("mean"), bias=c["b"], add=c["add"],
                             out_sum=got.get("s"), stream=stream) == 0
    return got


def run_norm_grad(train, c, x, rstd, mean, pad=0, dwt=F, base=None, stream=None):
    W = x.shape[-1]
    buf, dx = out_like(x.shape, x.dtype, pad)
    dw = torch.full((W,), 77.0, device=DEV, dtype=dwt) if base is None else base[0].clone()
    db = (torch.full((W,), 77.0, device=DEV, dtype=dwt) if base is None else base[1].clone()) if c["b"] is not None else None
    assert binding.mars_norm_grad(train, c["kind"], c["dy"], x, c["w"], rstd, dx, dw, mean=mean, db=db, d_sum=c["d_sum"],
                                  accumulate=base is not None, stream=stream) == 0
    return dict(dx=dx, dw=dw, db=db, buf=buf)


def check_norm(c, got, yt, pad):
    ref = norm_reference(c["kind"], c["x"], c["w"], c["b"], c["add"])
    assert worst(got["y"], ref["y"], rounded(yt, ref["y"], ref["tol"])) <= 1
    cols = math.prod(c["x"].shape[1:])
    assert (got["buf"][:, cols:] == 77).all()                    # what lies between the rows stays
    if "s" in got:
        assert torch.equal(got["s"], ref["s"]) and (got["s_buf"][:, cols:] == 77).all()
    if got.get("rstd") is not None:
        assert worst(got["rstd"], ref["rstd"], ref["tol_rstd"]) <= 1
    if got.get("mean") is not None:
        assert worst(got["mean"], ref["mean"], ref["tol_mean"] + V * ref["mean"].abs()) <= 1
    return ref


def check_norm_grad(c, got, x, rstd, mean, pad, base=None):
    ref = norm_grad_reference(c["kind"], c["dy"], x, c["w"], mean, rstd, c["d_sum"])
    assert worst(got["dx"], ref["dx"], rounded(x.dtype, ref["dx"], ref["tol_dx"])) <= 1
    assert (got["buf"][:, math.prod(x.shape[1:]):] == 77).all()
    for i, n in enumerate(("dw", "db")):
        if got[n] is not None:
            want = ref[n] + (0 if base is None else base[i].double())
            assert worst(got[n], want, rounded(got[n].dtype, want, ref["tol_" + n])) <= 1, n


SHAPES = [((1, 1), 0), ((3, 1), 2), ((2, 7), 0), ((5, 8), 0), ((33, 64), 8), ((4, 100), 4), ((9, 128), 0), ((70, 250), 1), ((300, 256), 8), ((17, 257), 0),
          ((31, 512), 0), ((6, 1000), 24), ((203, 1111), 0), ((40, 2048), 0), ((64, 2056), 8), ((5, 4096), 0), ((3, 5120), 0), ((2, 8191), 0),
          ((3, 8192), 8), ((2, 8184), 0), ((2, 6001), 1), ((40, 333), 0), ((500, 600), 1), ((31, 2500), 1), ((2000, 64), 0), ((7, 5, 128), 64), ((600, 32, 128), 0), ((4, 3, 50), 0), ((11, 1, 96), 8),
          ((9, 4, 640), 16)]


@pytest.mark.parametrize("shape,pad", SHAPES)
@pytest.mark.parametrize("kind", [RMS, LAYER])
def test_norms_and_their_gradients_match_the_formulas(shape, pad, kind):
    train = binding.Train(max_width=shape[-1], device=DEV)
    for i, (xt, yt, wt) in enumerate([(B, B, B), (F, F, F), (F, B, F), (H, H, B), (F, H, H)]):
        c = norm_case(kind, shape, xt, yt, wt, pad, seed=i, add=i % 2 == 0, bias=kind == LAYER and i != 3)
        got = run_norm(train, c, yt, pad)
        ref = check_norm(c, got, yt, pad)
        x = ref["s"]
        back = run_norm_grad(train, c, x, got["rstd"], got["mean"], pad)
        check_norm_grad(c, back, x, got["rstd"], got["mean"], pad)


@pytest.mark.parametrize("dwt", [F, B, H])
@pytest.mark.parametrize("shape", [(513, 264), (90, 1111)])
def test_weight_gradients_in_all_types_and_accumulated(dwt, shape):
    train = binding.Train(max_width=4096, device=DEV)            # a handle for wider rows
    c = norm_case(LAYER, shape, B, B, B, bias=True)
    got = run_norm(train, c, B)
    base = [normal(gen(9 + i), shape[1], dtype=dwt) for i in range(2)]
    for bs in (None, base):
        back = run_norm_grad(train, c, c["x"], got["rstd"], got["mean"], dwt=dwt, base=bs)
        check_norm_grad(c, back, c["x"], got["rstd"], got["mean"], 0, base=bs)


def test_norms_without_the_optional_parts():
    train = binding.Train(max_width=256, device=DEV)
    for kind in (RMS, LAYER):
        c = norm_case(kind, (50, 256), B, B, B)
        check_norm(c, run_norm(train, c, B, stats=False), B, 0)
        got = run_norm(train, c, B)
        dx, dw = torch.empty_like(c["x"]), torch.empty(256, device=DEV)
        full = run_norm_grad(train, c, c["x"], got["rstd"], got["mean"])
        assert binding.mars_norm_grad(train, kind, c["dy"], c["x"], c["w"], got["rstd"], dx, mean=got["mean"]) == 0
        assert torch.equal(dx, full["dx"])
        if kind == LAYER:
            db = torch.empty(256, device=DEV)
            assert binding.mars_norm_grad(train, kind, c["dy"], c["x"], c["w"], got["rstd"], dx, mean=got["mean"], db=db) == 0
            assert worst(db, c["dy"].double().sum(0), 400 * V * c["dy"].double().abs().sum(0)) <= 1
    # an addition whose sum is not kept
    c = norm_case(RMS, (50, 256), F, B, B, add=True)
    y = torch.empty(50, 256, device=DEV, dtype=B)
    assert binding.mars_norm(train, RMS, c["x"], c["w"], EPS, y, add=c["add"]) == 0
    assert torch.equal(y, run_norm(train, c, B)["y"])


def test_norms_in_place():
    train = binding.Train(max_width=2048, device=DEV)
    for width in (2048, 333):
        c = norm_case(RMS, (130, width), B, B, B, add=True)
        want = run_norm(train, c, B)
        back = run_norm_grad(train, c, want["s"], want["rstd"], None)
        x, add = c["x"].clone(), c["add"].clone()
        rstd = torch.empty(130, device=DEV)
        assert binding.mars_norm(train, RMS, x, c["w"], EPS, add, rstd=rstd, add=add, out_sum=x) == 0      # sum over x, y over add
        assert torch.equal(x, want["s"]) and torch.equal(add, want["y"]) and torch.equal(rstd, want["rstd"])
        for name in ("dy", "x", "d_sum"):
            a = dict(dy=c["dy"].clone(), x=want["s"].clone(), d_sum=c["d_sum"].clone())
            dw = torch.empty(width, device=DEV)
            assert binding.mars_norm_grad(train, RMS, a["dy"], a["x"], c["w"], rstd, a[name], dw, d_sum=a["d_sum"]) == 0
            assert torch.equal(a[name], back["dx"]) and torch.equal(dw, back["dw"])


def test_rows_beside_each_other_in_one_buffer():
    """q and k heads of a projection's rows, gradients into the same places of another buffer."""
    train = binding.Train(max_width=64, device=DEV)
    n, heads = 37, (6, 2)
    qkv, d_qkv = normal(gen(1), n, 12 * 64, dtype=B), torch.full((n, 12 * 64), 77.0, device=DEV, dtype=B)
    out = qkv.clone()
    at = 0
    for hs in heads:
        cut = lambda t: t[:, at:at + hs * 64].unflatten(1, (hs, 64))
        c = dict(kind=RMS, x=cut(qkv), w=normal(gen(hs), 64, dtype=B), b=None, add=None, d_sum=None, dy=cut(normal(gen(3 + hs), n, 12 * 64, dtype=B)))
        rstd, dw = torch.empty(n, hs, device=DEV), torch.empty(64, device=DEV)
        assert binding.mars_norm(train, RMS, cut(out), c["w"], EPS, cut(out), rstd=rstd) == 0
        ref = norm_reference(RMS, c["x"], c["w"], None)
        assert worst(cut(out), ref["y"], rounded(B, ref["y"], ref["tol"])) <= 1
        assert binding.mars_norm_grad(train, RMS, c["dy"], c["x"], c["w"], rstd, cut(d_qkv), dw) == 0
        back = norm_grad_reference(RMS, c["dy"], c["x"], c["w"], None, rstd)
        assert worst(cut(d_qkv), back["dx"], rounded(B, back["dx"], back["tol_dx"])) <= 1 and worst(dw, back["dw"], back["tol_dw"]) <= 1
        at += hs * 64
    assert torch.equal(out[:, at:], qkv[:, at:]) and (d_qkv[:, at:] == 77).all()


def test_norms_of_no_rows():
    train = binding.Train(max_width=64, device=DEV)
    e, s, w = torch.empty(0, 64, device=DEV), torch.empty(0, device=DEV), torch.ones(64, device=DEV)
    assert binding.mars_norm(train, LAYER, e, w, EPS, e, rstd=s, mean=s, bias=w) == 0
    dw, db = torch.ones(64, device=DEV), torch.ones(64, device=DEV)
    assert binding.mars_norm_grad(train, LAYER, e, e, w, s, e, dw, mean=s, db=db, accumulate=True) == 0
    assert (dw == 1).all() and (db == 1).all()
    assert binding.mars_norm_grad(train, LAYER, e, e, w, s, e, dw, mean=s, db=db) == 0
    assert (dw == 0).all() and (db == 0).all()


def test_rows_that_are_hard_for_norms():
    """Zeros, a constant row, a mean of a thousand spreads, large and tiny values."""
    train = binding.Train(max_width=520, device=DEV)
    g = gen(4)
    x = normal(g, 6, 520)
    x[0], x[1] = 0, 3.0
    x[2] = x[2] + 1000
    x[3] *= 1e15
    x[4] *= 1e-12
    w, b, dy = normal(g, 520, mean=1.0), normal(g, 520), normal(g, 6, 520)
    for kind in (RMS, LAYER):
        c = dict(kind=kind, x=x, w=w, b=b if kind == LAYER else None, add=None, d_sum=None, dy=dy)
        got = run_norm(train, c, F)
        assert torch.isfinite(got["y"]).all()
        check_norm(c, got, F, 0)
        check_norm_grad(c, run_norm_grad(train, c, x, got["rstd"], got["mean"]), x, got["rstd"], got["mean"], 0)
    # infinities and NaN stay in their rows
    bad = x.clone()
    bad[5, 17], bad[4, 3] = math.inf, math.nan
    got2 = run_norm(train, dict(c, x=bad), F)
    assert torch.equal(got2["y"][:4], got["y"][:4]) and got2["y"][4:].isnan().any(1).all()


def norm_loss(kind, x, w, b, up):
    d = x - (x.mean(-1, keepdim=True) if kind == LAYER else 0)
    y = d * (d.square().mean(-1, keepdim=True) + EPS).rsqrt() * w + (b if b is not None else 0)
    return (y * up).sum()


@pytest.mark.parametrize("kind", [RMS, LAYER])
def test_norm_gradients_against_differences(kind):
    train = binding.Train(max_width=72, device=DEV)
    c = norm_case(kind, (19, 72), F, F, F, bias=kind == LAYER)
    got = run_norm(train, c, F)
    back = run_norm_grad(train, c, c["x"], got["rstd"], got["mean"])
    g = gen(7)
    for name, key in (("x", "dx"), ("w", "dw"), ("b", "db")):
        if c[name] is None:
            continue
        at = {n: c[n].double() if c[n] is not None else None for n in ("x", "w", "b")}
        v = torch.randn(at[name].shape, generator=g, device=DEV, dtype=torch.float64)
        h = 1e-5
        f = [float(norm_loss(kind, *(dict(at, **{name: at[name] + s * h * v})[n] for n in ("x", "w", "b")), c["dy"].double())) for s in (1, -1)]
        along = float((back[key].double() * v).sum())
        # central differences: h^2 of a third derivative of order one, 1e-16 f / h; the gradient's own rounding V sqrt(n)
        assert abs((f[0] - f[1]) / (2 * h) - along) <= 1e-6 * (1 + abs(along)) * math.sqrt(v.numel())


# ---------------------------------------------------------------------------------------------- rotation

def rope_reference(x, positions, freq, rotary, layout, scale, inverse):
    a = positions.double()[:, None] * freq.to(DEV)
    c, s = (a.cos() * scale)[:, None], (a.sin() * scale * (-1 if inverse else 1))[:, None]
    d, out = x.double(), x.double().clone()
    h = rotary // 2
    i, j = (slice(0, h), slice(h, rotary)) if layout == "half" else (slice(0, rotary, 2), slice(1, rotary, 2))
    out[..., i], out[..., j] = d[..., i] * c - d[..., j] * s, d[..., j] * c + d[..., i] * s
    # sine and cosine: the fraction of a turn rounded to fp32 (2 pi 2^-26), two steps of the function, the product with scale
    tol = torch.zeros_like(d)
    both = (d[..., i].abs() + d[..., j].abs()) * scale * (2.0 ** -22 + 3 * V)
    tol[..., i], tol[..., j] = both, both
    return out, torch.where(tol > 0, rounded(x.dtype, out, tol), 0.0 * tol)


ROPES = [(1, 1, 0, 2, 2), (3, 2, 1, 8, 4), (17, 4, 1, 64, 64), (64, 32, 4, 128, 128), (33, 5, 2, 96, 64), (40, 3, 3, 80, 40), (9, 1, 1, 512, 512),
         (5, 2, 2, 510, 254), (257, 7, 0, 128, 96), (12, 64, 8, 64, 32), (2, 3, 0, 7, 6), (2100, 16, 2, 128, 128)]


@pytest.mark.parametrize("n,hq,hk,dim,rotary", ROPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotations_match_the_formula(n, hq, hk, dim, rotary, layout):
    for i, (t, pad, inverse) in enumerate([(B, 0, False), (B, 8, True), (F, 0, True), (H, 3, False), (F, 4, False)]):
        g = gen(n + i)
        scale = 1.0 if i % 2 else 1.2
        rope = binding.Rope(rotary, theta=1e4, layout=layout, scaling="linear" if i == 2 else "none", factor=4.0, scale=scale, device=DEV)
        positions = torch.randint(0, 1 << 20, (n,), generator=g, device=DEV, dtype=torch.int32)
        positions[0] = 0
        q, k = inside((n, hq, dim), t, g, pad)[1], inside((n, hk, dim), t, g, pad)[1] if hk else None
        bq, oq = out_like(q.shape, t, pad)
        bk, ok = out_like(k.shape, t, pad) if hk else (None, None)
        assert binding.mars_rope(rope, positions, q, oq, k, ok, inverse=inverse) == 0
        for x, o, buf in ((q, oq, bq), (k, ok, bk)):
            if x is None:
                continue
            want, tol = rope_reference(x, positions, rope.frequencies(), rotary, layout, float(torch.tensor(scale)), inverse)
            assert worst(o, want, tol) <= 1
            assert (buf[:, x.shape[1] * dim:] == 77).all()
            # in place
            same = x.clone(memory_format=torch.contiguous_format)
            assert binding.mars_rope(rope, positions, same, same, inverse=inverse) == 0 and torch.equal(same, o)


@pytest.mark.parametrize("n,hq,hk,dim,t", [(9001, 32, 4, 128, B), (5003, 37, 3, 64, H), (3001, 20, 0, 90, F), (70001, 5, 1, 64, B)])
def test_rotations_of_many_rows(n, hq, hk, dim, t):
    """One, two and three rounds of heads for a thread, heads left over among them."""
    for layout in ("half", "interleaved"):
        g = gen(n)
        rope = binding.Rope(dim // 2 * 2, theta=1e4, layout=layout, device=DEV)
        positions = torch.randint(0, 1 << 15, (n,), generator=g, device=DEV, dtype=torch.int32)
        for h in (hq, hk):
            if h:
                x = normal(g, n, h, dim).to(t)
                o = torch.empty_like(x)
                other = normal(g, n, hq + hk - h, dim).to(t) if hk else None
                back = torch.empty_like(other) if hk else None
                assert binding.mars_rope(rope, positions, x, o, other, back) == 0
                for got, src in ((o, x), (back, other)):
                    if src is not None:
                        want, tol = rope_reference(src, positions, rope.frequencies(), dim // 2 * 2, layout, 1.0, False)
                        assert worst(got, want, tol) <= 1


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
def test_far_positions_keep_their_angles(scaling):
    """The largest and smallest positions, against cosines of a reduced angle in whole-number arithmetic."""
    rope = binding.Rope(64, theta=1e6, scaling=scaling, factor=8.0, trained_positions=32768, device=DEV)
    positions = torch.tensor([0, 1, 32767, 1_000_003, 2 ** 31 - 1, -2 ** 31, -5], dtype=torch.int32, device=DEV)
    x = torch.zeros(7, 1, 64, device=DEV)
    x[..., :32] = 1                                              # (1, 0) turns to (cos, sin)
    out = torch.empty_like(x)
    assert binding.mars_rope(rope, positions, x, out) == 0
    freq = rope.frequencies()
    for i, p in enumerate(positions.tolist()):
        for j in range(32):
            a = math.fmod(p * float(freq[j]), 2 * math.pi)       # p x frequency rounds in its 53rd bit: 2e9 turns 5e-7 off at most
            e = 2.0 ** -22 + 2 * abs(p) * float(freq[j]) * 2.0 ** -52
            assert abs(float(out[i, 0, j]) - math.cos(a)) <= e and abs(float(out[i, 0, 32 + j]) - math.sin(a)) <= e


def test_a_rotation_and_back_is_the_identity_and_its_gradient():
    rope = binding.Rope(128, device=DEV)
    g = gen(3)
    positions = torch.randint(0, 65536, (50,), generator=g, device=DEV, dtype=torch.int32)
    q, up = normal(g, 50, 4, 128), normal(g, 50, 4, 128)
    o, back, d = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    assert binding.mars_rope(rope, positions, q, o) == 0 and binding.mars_rope(rope, positions, o, back, inverse=True) == 0
    assert float((back - q).abs().max()) <= 2 ** -20 * float(q.abs().max()) * 2
    assert binding.mars_rope(rope, positions, up, d, inverse=True) == 0
    # differences of sum(up rotated(q)) along a direction (the map is linear: any step does)
    rot = lambda t: rope_reference(t.float(), positions, rope.frequencies(), 128, "half", 1.0, False)[0]
    v = normal(g, *q.shape)
    along = float(((rot(q + v) - rot(q - v)) / 2 * up.double()).sum())
    got = float((d.double() * v.double()).sum())
    assert abs(along - got) <= 2.0 ** -20 * float(up.double().norm() * v.double().norm()) * 2


def test_q_and_k_in_the_rows_of_one_projection_in_place():
    rope = binding.Rope(64, device=DEV)
    n, g = 77, gen(5)
    qkv = normal(g, n, 8 * 64, dtype=B)
    positions = torch.arange(n, device=DEV, dtype=torch.int32)
    old = qkv.clone()
    q, k = qkv[:, :5 * 64].unflatten(1, (5, 64)), qkv[:, 5 * 64:6 * 64].unflatten(1, (1, 64))
    assert binding.mars_rope(rope, positions, q, q, k, k) == 0
    want, tol = rope_reference(old[:, :6 * 64].unflatten(1, (6, 64)), positions, rope.frequencies(), 64, "half", 1.0, False)
    assert worst(qkv[:, :6 * 64].unflatten(1, (6, 64)), want, tol) <= 1 and torch.equal(qkv[:, 6 * 64:], old[:, 6 * 64:])
    e = torch.empty(0, 5, 64, dtype=B, device=DEV)
    assert binding.mars_rope(rope, positions[:0], e, e) == 0


# ------------------------------------------------------------------------------------------------ router

def router_reference(z, k, live, renormalise):
    d = z.double()
    n, E = d.shape
    on = ((d != -math.inf).any(1)) if live is None else live & (d != -math.inf).any(1)
    lse = torch.where(on, torch.logsumexp(torch.where(on[:, None], d, 0.0), 1), 0.0)
    p = torch.where(on[:, None], (d - lse[:, None]).exp(), 0.0)
    idx = torch.sort(torch.where(on[:, None], d, 0.0), dim=1, descending=True, stable=True).indices[:, :k]
    w = p.gather(1, idx)
    if renormalise:
        w = w / w.sum(1, keepdim=True)
    w = torch.where(on[:, None], w, 0.0)
    counts = torch.bincount(idx[on].flatten(), minlength=E)
    N = int(on.sum())
    sums = p.sum(0)
    balance = E * float((counts.double() * sums).sum()) / max(1, N) ** 2 / k if N else 0.0
    zl = float((lse ** 2).sum()) / N if N else 0.0
    # relative error of an exponential whose argument z - max (or z - lse) is rounded, of the sum of E of them and the quotient
    far = torch.where(torch.isfinite(d) & on[:, None], (d - lse[:, None]).abs(), 0.0)
    rel = 64 * V + 2 * V * far.max(1).values + 2 * V * lse.abs()
    return dict(on=on, lse=lse, p=p, idx=torch.where(on[:, None], idx, -1), w=w, counts=counts, sums=sums, N=N, rel=rel,
                losses=torch.tensor([balance, zl], dtype=torch.float64, device=DEV))


def run_router(train, z, k, live=None, renormalise=True, stream=None):
    n, E = z.shape
    i32 = dict(device=DEV, dtype=torch.int32)
    got = dict(idx=torch.full((n, k), 77, **i32), w=torch.full((n, k), 77.0, device=DEV), lse=torch.full((n,), 77.0, device=DEV),
               counts=torch.full((E,), 77, **i32), off=torch.full((E + 1,), 77, **i32), sums=torch.full((E,), 77.0, device=DEV),
               losses=torch.full((2,), 77.0, device=DEV))
    assert binding.mars_router(train, z, got["idx"], got["w"], got["lse"], got["counts"], got["off"], got["sums"], got["losses"], live=live,
                               renormalise=renormalise, stream=stream) == 0
    return got


def check_router(z, k, got, live=None, renormalise=True):
    ref = router_reference(z, k, live, renormalise)
    assert torch.equal(got["idx"].long(), ref["idx"])
    assert torch.equal(got["counts"].long(), ref["counts"])
    assert torch.equal(got["off"].long(), torch.cat([ref["counts"].new_zeros(1), ref["counts"].cumsum(0)]))
    rel = ref["rel"]
    assert worst(got["w"], ref["w"], 2 * rel[:, None] * ref["w"] + 1e-45) <= 1
    assert worst(got["lse"], ref["lse"], rel + V * ref["lse"].abs()) <= 1
    # sums: rows of a warp (148 blocks of 8 warps at least), warps of a block; the blocks in fp64
    chain = z.shape[0] / 1184 + 34
    assert worst(got["sums"], ref["sums"], ref["sums"] * (float(rel.max()) + chain * V) + 1e-40) <= 1
    most = 2 * float(rel.max()) + (chain + 4) * V
    lse2 = float((ref["lse"].abs() * (rel + V * ref["lse"].abs())).sum()) * 2 / max(1, ref["N"])
    assert abs(float(got["losses"][0]) - float(ref["losses"][0])) <= most * float(ref["losses"][0])
    if float(ref["losses"][1]) > torch.finfo(F).max * (1 + V):   # the squares of lowest values: beyond fp32, rounded to infinity
        assert float(got["losses"][1]) == math.inf
    else:
        assert abs(float(got["losses"][1]) - float(ref["losses"][1])) <= lse2 + 2 * V * float(ref["losses"][1])
    return ref


def router_logits(n, E, t, seed=0, pad=0, std=1.3):
    g = gen(seed)
    buf = torch.full((n, E + pad), math.nan, device=DEV, dtype=t)
    buf[:, :E] = (normal(g, n, E, std=std) + normal(g, E, std=0.5)).to(t)
    return buf[:, :E]


ROUTERS = [(1, 1, 1, 0), (1, 8, 2, 0), (3, 2, 2, 0), (64, 128, 8, 0), (65, 128, 8, 4), (100, 60, 4, 0), (1000, 64, 6, 0), (37, 127, 8, 1), (16, 129, 8, 3),
           (50, 256, 8, 0), (21, 300, 10, 0), (33, 512, 16, 8), (12, 1024, 32, 0), (9, 1023, 32, 0), (5000, 128, 8, 0), (40, 32, 32, 0), (7, 16, 1, 0)]


@pytest.mark.parametrize("n,E,k,pad", ROUTERS)
@pytest.mark.parametrize("t", [F, B, H])
def test_router_and_gradient_match_the_formulas(n, E, k, pad, t):
    train = binding.Train(max_experts=E, device=DEV)
    for renormalise, masked in ((True, False), (False, True)):
        z = router_logits(n, E, t, seed=n + E, pad=pad)
        live = torch.rand(n, generator=gen(2), device=DEV) < 0.6 if masked else None
        if live is not None:
            z[~live] = math.nan                                  # padding may hold anything
        got = run_router(train, z, k, live, renormalise)
        check_router(z, k, got, live, renormalise)
        dw = normal(gen(5), n, k)
        if live is not None:
            dw[~live] = math.nan
        check_router_grad(train, z, k, got, dw, renormalise, 0.7, 0.03)
        check_router_grad(train, z, k, got, None, renormalise, 0.7, 0.0)
        check_router_grad(train, z, k, got, dw, renormalise, 0.0, 0.0)


def check_router_grad(train, z, k, got, dw, renormalise, cb, cz):
    n, E = z.shape
    buf = torch.full((n, E + 4), 77.0, device=DEV, dtype=z.dtype)
    d = buf[:, :E]
    assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], d, d_weights=dw, balance_coef=cb, z_coef=cz,
                                    renormalise=renormalise) == 0
    want, tol = router_grad_reference(z, k, got, dw, renormalise, cb, cz)
    assert worst(d, want, rounded(z.dtype, want, tol)) <= 1
    assert (buf[:, E:] == 77).all()


def router_grad_reference(z, k, got, dw, renormalise, cb, cz):
    n, E = z.shape
    on = got["idx"][:, 0] >= 0
    lse = got["lse"].double()
    p = torch.where(on[:, None], (z.double() - lse[:, None]).exp(), 0.0)
    total = float(got["counts"].sum())
    N = max(1.0, total / k)
    g = cb * E / N * got["counts"].double() / max(1.0, total)
    dot = (p * g).sum(1, keepdim=True)
    want = p * (g - dot + 2 * cz / N * lse[:, None])
    scale = p * (g.abs() + (p * g.abs()).sum(1, keepdim=True) + (2 * cz / N * lse[:, None]).abs())
    if dw is not None:
        at, dwd = got["idx"].clamp(min=0).long(), torch.where(on[:, None], dw.double(), 0.0)
        sel = p.gather(1, at)
        if renormalise:
            w = torch.where(on[:, None], sel / sel.sum(1, keepdim=True), 0.0)
            push = w * (dwd - (w * dwd).sum(1, keepdim=True))
            size = w * (dwd.abs() + (w * dwd.abs()).sum(1, keepdim=True))
        else:
            push, size = sel * dwd, sel * dwd.abs()
            want = want - p * (sel * dwd).sum(1, keepdim=True)
            scale = scale + p * (sel * dwd.abs()).sum(1, keepdim=True)
        want, scale = want.scatter_add(1, at, torch.where(on[:, None], push, 0.0)), scale.scatter_add(1, at, torch.where(on[:, None], size, 0.0))
    far = torch.where(on[:, None] & torch.isfinite(z.double()), (z.double() - lse[:, None]).abs(), 0.0).max(1).values[:, None]
    # exponentials (argument rounded), sums over 1024 experts in chains of 64 and the products
    return want, scale * (128 + 4 * far) * V + 1e-45


@pytest.mark.parametrize("E,k", [(2, 2), (8, 8), (9, 1), (60, 4), (61, 5), (64, 6), (128, 8), (129, 3), (250, 8), (256, 7), (256, 10), (300, 8), (384, 6), (511, 8), (512, 8), (513, 8)])
@pytest.mark.parametrize("t", [F, B, H])
def test_router_of_many_rows(E, k, t):
    n = 8192 + 77
    train = binding.Train(max_experts=E, device=DEV)
    for renormalise, masked, pad in ((True, False, 0), (False, True, 4 if E % 4 == 0 else 1)):
        z = router_logits(n, E, t, seed=E, pad=pad)
        z[5, :] = -math.inf
        z[6, 1:] = -math.inf
        z[7, :] = 0.5
        z[8, : E // 2] = torch.finfo(t).min
        live = torch.rand(n, generator=gen(2), device=DEV) < 0.6 if masked else None
        if live is not None:
            live[5:9] = True
            z[~live] = math.nan
        got = run_router(train, z, k, live, renormalise)
        check_router(z, k, got, live, renormalise)
        again = run_router(train, z, k, live, renormalise)
        assert all(torch.equal(got[n_], again[n_]) for n_ in got if n_ != "losses")


@pytest.mark.parametrize("E", [64, 128, 200, 512])
def test_logits_that_differ_in_their_last_bits(E):
    """fp32 logits whose leading bits agree: the order is that of the values, not of the leading bits."""
    n, k = 9000, 8
    train = binding.Train(max_experts=E, device=DEV)
    g = gen(9)
    steps = torch.randint(0, 200, (n, E), generator=g, device=DEV)
    z = (torch.tensor(2.5, device=DEV).view(torch.int32) + steps.int()).view(F)      # 2.5 and the 199 numbers after it, ties among them
    z[::3] = -z[::3]
    z[1::7] = router_logits(len(z[1::7]), E, F)
    z[2::5, E - 28:] = z[2::5, :28]                              # pairs of equal logits
    got = run_router(train, z, k)
    check_router(z, k, got)
    z[17, 3], z[18, 60], z[19, 5], z[20, :], z[21, 2:] = math.nan, math.inf, -math.nan, math.nan, -math.nan
    bad = run_router(train, z, k)
    keep = torch.ones(n, dtype=torch.bool, device=DEV)
    keep[17:22] = False
    assert torch.equal(bad["idx"][keep], got["idx"][keep]) and torch.equal(bad["w"][keep], got["w"][keep])
    for row in bad["idx"][17:22].tolist():
        assert len(set(row)) == k and min(row) >= 0 and max(row) < E
    assert bad["w"][17:22].isnan().any(1).all()


def test_equal_logits_go_to_the_lower_expert():
    for E in (8, 128, 130, 600):
        train = binding.Train(max_experts=E, device=DEV)
        z = torch.randint(-2, 3, (300, E), generator=gen(E), device=DEV).to(B)
        z[0] = 0
        z[1] = torch.where(torch.arange(E, device=DEV) % 2 == 0, 0.0, -0.0)      # -0 and 0 are equal
        got = run_router(train, z, 8)
        check_router(z, 8, got)
        assert got["idx"][0].tolist() == list(range(8)) and got["idx"][1].tolist() == list(range(8))


@pytest.mark.parametrize("E", [16, 128, 200])
def test_experts_and_rows_that_are_shut_out(E):
    """-inf and the type's lowest value on some experts, on all but a few, and on whole rows; +inf and NaN stay in their row."""
    train = binding.Train(max_experts=E, device=DEV)
    k = 6
    for t in (F, B):
        z = router_logits(40, E, t, seed=3)
        z[0, :] = -math.inf                                      # nothing left: takes no part
        z[1, 3:] = -math.inf                                     # fewer than k left
        z[2, 1:] = torch.finfo(t).min
        z[3, :] = torch.finfo(t).min
        z[4, ::2] = -math.inf
        z[5, 7] = 1000.0
        got = run_router(train, z, k)
        ref = check_router(z, k, got)
        assert not ref["on"][0] and got["idx"][1].tolist() == sorted(got["idx"][1][:3].tolist(), key=lambda e: -float(z[1, e])) + [3, 4, 5]
        assert (got["idx"][0] == -1).all() and (got["w"][0] == 0).all() and got["lse"][0] == 0 and got["idx"][3].tolist() == list(range(k))
        check_router_grad(train, z, k, got, normal(gen(1), 40, k), True, 0.5, 0.01)
        z2 = z.clone()
        z2[39, 5], z2[38, 9] = math.nan, math.inf
        bad = run_router(train, z2, k)
        assert torch.equal(bad["idx"][:38], got["idx"][:38]) and torch.equal(bad["w"][:38], got["w"][:38])
        assert bad["w"][38:].isnan().any(1).all()
        for row in bad["idx"][38:].tolist():
            assert len(set(row)) == k and min(row) >= 0 and max(row) < E


def test_router_of_no_rows_and_of_padding_alone():
    train = binding.Train(max_experts=20, device=DEV)
    for n in (0, 50):
        z = router_logits(n, 20, F)
        got = run_router(train, z, 3, torch.zeros(n, dtype=torch.bool, device=DEV))
        assert (got["counts"] == 0).all() and (got["off"] == 0).all() and (got["sums"] == 0).all() and (got["losses"] == 0).all()
        assert (got["idx"] == -1).all() and (got["w"] == 0).all() and (got["lse"] == 0).all()
        d = torch.full((n, 20), 77.0, device=DEV)
        assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], d, balance_coef=1.0, z_coef=1.0) == 0
        assert (d == 0).all()


def test_router_without_the_optional_outputs_and_in_place():
    train = binding.Train(max_experts=64, device=DEV)
    z = router_logits(90, 64, B)
    full = run_router(train, z, 4)
    idx, w = torch.empty_like(full["idx"]), torch.empty_like(full["w"])
    assert binding.mars_router(train, z, idx, w) == 0
    assert torch.equal(idx, full["idx"]) and torch.equal(w, full["w"])
    dw = normal(gen(1), 90, 4)
    d = torch.empty_like(z)
    assert binding.mars_router_grad(train, z, idx, full["lse"], full["counts"], d, d_weights=dw, balance_coef=0.2) == 0
    same = z.clone()
    assert binding.mars_router_grad(train, same, idx, full["lse"], full["counts"], same, d_weights=dw, balance_coef=0.2) == 0
    assert torch.equal(same, d)


def test_gradient_of_choices_that_are_not_the_routers():
    """Indexes outside the experts are left out; the same expert twice counts twice."""
    train = binding.Train(max_experts=12, device=DEV)
    z = router_logits(3, 12, F)
    got = run_router(train, z, 3)
    idx = torch.tensor([[2, 99, 5], [4, 4, 7], [0, -3, 11]], dtype=torch.int32, device=DEV)
    dw = normal(gen(1), 3, 3)
    d = torch.empty_like(z)
    assert binding.mars_router_grad(train, z, idx, got["lse"], got["counts"], d, d_weights=dw) == 0
    keep = (idx >= 0) & (idx < 12)
    sel = torch.where(keep, torch.softmax(z.double(), 1).gather(1, idx.clamp(0, 11).long()), 0.0)
    w = sel / sel.sum(1, keepdim=True)
    push = w * (dw.double() - (w * dw.double()).sum(1, keepdim=True))
    want = torch.zeros(3, 12, dtype=torch.float64, device=DEV).scatter_add_(1, idx.clamp(0, 11).long(), torch.where(keep, push, 0.0))
    assert float((d.double() - want).abs().max()) <= 256 * V * float(dw.abs().max())


@pytest.mark.parametrize("E,k,t", [(20, 3, F), (32, 8, B), (61, 5, H), (128, 8, B), (128, 12, F), (200, 8, H), (384, 6, F), (600, 4, B), (602, 10, F)])
def test_router_gradient_of_many_rows(E, k, t):
    """More rows than are on their way at once, rows that take no part among them, in place of the logits as well."""
    n = 60011
    train = binding.Train(max_experts=E, device=DEV)
    z = router_logits(n, E, t, seed=E, pad=4)
    live = torch.rand(n, generator=gen(2), device=DEV) < 0.9
    z[~live] = math.nan
    got = run_router(train, z, k, live, True)
    dw = normal(gen(5), n, k)
    dw[~live] = math.nan
    check_router_grad(train, z, k, got, dw, True, 0.7, 0.03)
    d, same = torch.empty(n, E, dtype=t, device=DEV), z.clone()
    assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], d, d_weights=dw, balance_coef=0.7) == 0
    assert binding.mars_router_grad(train, same, got["idx"], got["lse"], got["counts"], same, d_weights=dw, balance_coef=0.7) == 0
    assert torch.equal(same, d)
    # one expert twice: as if it were chosen once with the mean of both gradients and twice the weight
    twice, once = got["idx"][:, :1].repeat(1, 2), got["idx"][:, :1].contiguous()
    pair, mean = dw[:, :2].contiguous(), dw[:, :2].double().sum(1, keepdim=True).float()
    a, b = (torch.empty(n, E, dtype=t, device=DEV) for _ in range(2))
    assert binding.mars_router_grad(train, z, twice, got["lse"], got["counts"], a, d_weights=pair, renormalise=False) == 0
    assert binding.mars_router_grad(train, z, once, got["lse"], got["counts"], b, d_weights=mean, renormalise=False) == 0
    # both are p_j ([chosen] sum of dw - p sum of dw) of the same exponentials: some ten roundings of terms of at most |dw1| + |dw2|, and
    # each result's own
    size = pair.double().abs().sum(1, keepdim=True).nan_to_num() * 16 * V
    assert worst(a, b.double(), rounded(t, b.double(), size) + U[t] * b.double().abs() + 1e-45) <= 1


@pytest.mark.parametrize("E,k", [(16, 1), (128, 2), (128, 8)])
def test_weights_next_to_one_keep_their_gradients_accuracy(E, k):
    """Renormalised weights: a first choice that leaves the others 1e-2 .. 1e-9, or that is the only one (no gradient at all)."""
    n = 64
    train = binding.Train(max_experts=E, device=DEV)
    z = router_logits(n, E, F, seed=2, std=0.3)
    z[torch.arange(n), torch.arange(n) % E] += torch.linspace(5.0, 20.0, n, device=DEV)
    got = run_router(train, z, k)
    dw = normal(gen(5), n, k, mean=3.0)
    d = torch.empty_like(z)
    assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], d, d_weights=dw) == 0
    at = got["idx"].long()
    sel = z.double().gather(1, at)
    w = torch.softmax(sel, 1)
    # w_i sum_j w_j (dw_i - dw_j): no difference of nearly equal numbers but those of the inputs
    diff = dw.double()[:, :, None] - dw.double()[:, None, :]
    push = w * (w[:, None, :] * diff).sum(2)
    size = w * (w[:, None, :] * diff.abs()).sum(2)
    want = torch.zeros(n, E, dtype=torch.float64, device=DEV).scatter_(1, at, push)
    # exponentials of rounded arguments (up to 25), 8 of them added, products and differences of a few roundings
    tol = torch.zeros_like(want).scatter_(1, at, size) * (64 + 4 * 25) * V
    assert worst(d, want, tol + 1e-45) <= 1


def test_counts_of_several_micro_batches():
    """counts added up: each call's gradient is its rows' share of the gradient over all rows."""
    train = binding.Train(max_experts=40, device=DEV)
    z = router_logits(300, 40, F, seed=8)
    whole = run_router(train, z, 4)
    want = torch.empty_like(z)
    assert binding.mars_router_grad(train, z, whole["idx"], whole["lse"], whole["counts"], want, balance_coef=0.3, z_coef=0.1) == 0
    parts = [run_router(train, z[a:b], 4) for a, b in ((0, 77), (77, 300))]
    counts = parts[0]["counts"] + parts[1]["counts"]
    assert torch.equal(counts, whole["counts"])
    for p, (a, b) in zip(parts, ((0, 77), (77, 300))):
        d = torch.empty_like(z[a:b])
        assert binding.mars_router_grad(train, z[a:b], p["idx"], p["lse"], counts, d, balance_coef=0.3, z_coef=0.1) == 0
        assert torch.equal(d, want[a:b])


@pytest.mark.parametrize("renormalise", [True, False])
def test_router_gradient_against_differences(renormalise):
    n, E, k, cb, cz = 25, 24, 3, 0.5, 0.2
    train = binding.Train(max_experts=E, device=DEV)
    z = router_logits(n, E, F, seed=11)
    got = run_router(train, z, k, renormalise=renormalise)
    dw = normal(gen(3), n, k)
    d = torch.empty_like(z)
    assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], d, d_weights=dw, balance_coef=cb, z_coef=cz,
                                    renormalise=renormalise) == 0
    at, f = got["idx"].long(), got["counts"].double() / (n * k)

    def loss(t):
        p = torch.softmax(t, 1)
        w = p.gather(1, at)
        w = w / w.sum(1, keepdim=True) if renormalise else w
        return float((w * dw.double()).sum() + cb * E * (f * p.mean(0)).sum() + cz * torch.logsumexp(t, 1).square().mean())

    for seed in range(3):
        v = torch.randn(z.shape, generator=gen(seed), device=DEV, dtype=torch.float64)
        h = 1e-5
        num = (loss(z.double() + h * v) - loss(z.double() - h * v)) / (2 * h)
        along = float((d.double() * v).sum())
        assert abs(num - along) <= 1e-6 * (1 + abs(along)) * math.sqrt(n)


# ------------------------------------------------------------------------------------------- policy loss

def policy_reference(c, low, high, kl, reduce, scale, per_token):
    off = c["off"].tolist()
    n = c["lp"].shape[0]
    seq = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    for s in range(len(off) - 1):
        seq[max(0, off[s]):min(n, off[s + 1])] = s
    on = (c["t"] >= 0) & (seq >= 0)
    held = torch.bincount(seq[on], minlength=len(off) - 1).double()
    live, seqs = float(held.sum()), float((held > 0).sum())
    share = torch.zeros(n, dtype=torch.float64, device=DEV)
    if reduce == "tokens":
        share[on] = scale / live if live else 0.0
    elif reduce == "sequences":
        share[on] = scale / (held[seq[on]] * seqs)
    else:
        share[on] = scale
    zero = torch.zeros(n, dtype=torch.float64, device=DEV)
    sel = lambda t: torch.where(on, t.double(), zero)
    lp, old = sel(c["lp"]), sel(c["old"])
    A = torch.where(on, c["adv"].double() if per_token else c["adv"].double()[seq.clamp(min=0)], zero)
    r = (lp - old).exp()
    first, second = r * A, r.clamp(1 - low, 1 + high) * A
    cut = (second < first) & on
    term, d = -torch.minimum(first, second), torch.where(cut, zero, -first)
    x = sel(c["ref"]) - lp if c["ref"] is not None else zero
    em1, kls = x.expm1(), x.expm1() - x
    term, d = term + kl * kls, d - kl * em1
    x_d = (lp - old).abs()
    # exp of a rounded argument, products; expm1 the same; exp(x) - 1 - x by its series (|x| < 1/2) or as a difference
    e_r = (x_d + 8) * V * (r * A).abs()
    e_em1 = V * (4 * em1.abs() + 2 * x.abs() * x.exp())
    e_kl = torch.where(x.abs() < 0.5, 12 * V * kls, V * (5 * em1.abs() + 2 * x.abs() * x.exp() + 2 * x.abs()))
    count = max(1.0, live)
    stats = torch.stack([(share * term).sum(), sel(kls).sum() / count, cut.double().sum() / count, sel(r).sum() / count,
                         torch.tensor(live, device=DEV, dtype=torch.float64), torch.tensor(seqs, device=DEV, dtype=torch.float64)])
    tol_s = torch.stack([(share.abs() * (e_r + V * first.abs() + V * second.abs() + kl * e_kl + 3 * V * kl * kls)).sum(), sel(e_kl).sum() / count, 0 * zero.sum(),
                         sel((x_d + 8) * V * r).sum() / count, 0 * zero.sum(), 0 * zero.sum()])
    return dict(stats=stats, tol_stats=tol_s + V * stats.abs(), d=share * d, tol_d=share.abs() * (e_r + kl * e_em1 + 4 * V * (first.abs() + kl * em1.abs())) +
                2 * V * (share * d).abs() + 1e-45)


def policy_case(lengths, masked=0.3, ref=True, per_token=False, seed=0, before=0, behind=0):
    g = gen(seed)
    n = sum(lengths) + before + behind
    off = torch.tensor([before] + [before + sum(lengths[:i + 1]) for i in range(len(lengths))], dtype=torch.int32, device=DEV)
    old = -normal(g, n).abs() ** 3 * 0.5
    lp = (old + normal(g, n) * 0.3).clamp(max=0)
    t = torch.randint(0, 1000, (n,), generator=g, device=DEV, dtype=torch.int32)
    t[torch.rand(n, generator=g, device=DEV) < masked] = -1
    c = dict(lp=lp, old=old, t=t, off=off, adv=normal(g, n if per_token else len(lengths)), ref=lp + normal(g, n) * 0.4 if ref else None)
    if before:
        t[:before] = 5
    if behind:
        t[n - behind:] = 5
    dead = t < 0
    dead[:before] = True
    dead[n - behind:] = True if behind else dead[n - behind:]
    for name in ("lp", "old", "ref"):
        if c[name] is not None:
            c[name][dead] = math.nan                             # tokens that take no part may hold anything
    if per_token:
        c["adv"][dead] = math.nan
    return c


def run_policy(train, c, low=0.2, high=0.28, kl=0.0, reduce="tokens", scale=1.0, per_token=False, stream=None):
    stats, d = torch.full((6,), 77.0, device=DEV), torch.full_like(c["lp"], 77.0)
    assert binding.mars_policy_loss(train, c["lp"], c["old"], c["adv"], c["t"], c["off"], stats, d, ref_logprobs=c["ref"], clip_low=low,
                                    clip_high=high, kl_coef=kl, reduce=reduce, scale=scale, per_token=per_token, stream=stream) == 0
    return dict(stats=stats, d=d)


def check_policy(c, got, low=0.2, high=0.28, kl=0.0, reduce="tokens", scale=1.0, per_token=False):
    ref = policy_reference(c, low, high, kl, reduce, scale, per_token)
    assert worst(got["stats"], ref["stats"], ref["tol_stats"]) <= 1, (got["stats"], ref["stats"])
    assert worst(got["d"], ref["d"], ref["tol_d"]) <= 1
    return ref


LENGTHS = [[1], [5], [3, 4, 0, 1], [1023, 1, 1024], [1024, 1024], [0, 0, 7, 0], [700, 2000, 31, 5, 0, 900], [1] * 2500, [0] * 600 + [50] + [0] * 600,
           [70000], [4097] * 9, [1025, 3, 0] * 40, [2] * 300 + [3000] + [0] * 300]


@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: f"{len(v)}x{sum(v)}")
@pytest.mark.parametrize("reduce", ["tokens", "sequences", "sum"])
def test_policy_loss_and_gradient_match_the_formula(lengths, reduce):
    train = binding.Train(max_seqs=len(lengths), device=DEV)
    for kl, ref, per_token, before, behind in ((0.0, False, False, 0, 0), (0.05, True, True, 0, 0), (0.001, True, False, 13, 2001)):
        c = policy_case(lengths, ref=ref, per_token=per_token, seed=len(lengths), before=before, behind=behind)
        kw = dict(kl=kl, reduce=reduce, scale=1.0 if reduce != "sum" else 0.01, per_token=per_token)
        check_policy(c, run_policy(train, c, **kw), **kw)


@pytest.mark.parametrize("low,high", [(1.0, 0.2), (0.2, 1e6), (0.0, 0.0), (0.2, 0.28)])
def test_policy_loss_of_zero_advantages_and_open_borders(low, high):
    train = binding.Train(max_seqs=9, device=DEV)
    for reduce, kl in (("sequences", 0.0), ("tokens", 0.3)):
        c = policy_case([2000, 150, 1, 4000, 0, 700, 128, 128, 3000], masked=0.1, seed=4)
        c["adv"][::2] = 0.0
        c["adv"][1] = -1e-40
        c["ref"] = c["lp"] + normal(gen(1), c["lp"].shape[0], std=1.0)           # many differences beyond 1/2
        kw = dict(low=low, high=high, kl=kl, reduce=reduce)
        ref = check_policy(c, run_policy(train, c, **kw), **kw)
        assert float(ref["stats"][2]) > 0 or high > 1 or low == 1.0


def test_policy_loss_without_live_tokens_and_without_tokens():
    train = binding.Train(max_seqs=4, device=DEV)
    for reduce in ("tokens", "sequences", "sum"):
        c = policy_case([5, 0, 9], masked=1.1)
        got = run_policy(train, c, kl=0.1, reduce=reduce)
        assert (got["stats"] == 0).all() and (got["d"] == 0).all()
        c = policy_case([0, 0, 0])
        got = run_policy(train, c, reduce=reduce)
        assert (got["stats"] == 0).all()


def test_ratios_at_the_borders():
    """Which side of a border a ratio is on is decided exactly; at the border itself the gradient is that of r A."""
    low, high = 0.25, 0.25
    steps = []
    for b in (math.log(0.75), math.log(1.25)):
        f = torch.tensor(b, dtype=F)
        steps += [float(f), float(torch.nextafter(f, torch.tensor(9.0))), float(torch.nextafter(f, torch.tensor(-9.0)))]
    lp = torch.tensor(steps + steps + [0.0, 0.0], device=DEV)
    n = lp.shape[0]
    c = dict(lp=lp, old=torch.zeros(n, device=DEV), t=torch.zeros(n, dtype=torch.int32, device=DEV), ref=None,
             off=torch.tensor([0, n], dtype=torch.int32, device=DEV), adv=torch.tensor([1.0] * 6 + [-1.0] * 6 + [2.0, -2.0], device=DEV))
    train = binding.Train(max_seqs=1, device=DEV)
    got = run_policy(train, c, low=low, high=high, per_token=True)
    ref = check_policy(c, got, low=low, high=high, per_token=True)
    assert torch.equal(got["d"] == 0, ref["d"] == 0) and 0 < int((got["d"] == 0).sum()) < 12
    # no border below (clip_low 1) and none of either (a wide clip): every gradient flows
    got = run_policy(train, c, low=1.0, high=10.0, per_token=True)
    assert (got["d"] != 0).all()
    # a clip of nothing: the ratio 1 itself is not cut
    got = run_policy(train, c, low=0.0, high=0.0, per_token=True)
    assert (got["d"][-2:] != 0).all()
    check_policy(c, got, low=0.0, high=0.0, per_token=True)


def test_infinite_log_probs():
    """logp = -inf: ratio 0; old = -inf: an infinite ratio that is cut for A > 0; tiny and huge KL arguments."""
    n = 6
    c = dict(lp=torch.tensor([-math.inf, -1.0, -1.0, -1.0, -50.0, -1e-4], device=DEV), old=torch.tensor([-1.0, -math.inf, -1.0, -30.0, -1.0, -2e-4], device=DEV),
             t=torch.zeros(n, dtype=torch.int32, device=DEV), off=torch.tensor([0, n], dtype=torch.int32, device=DEV),
             adv=torch.tensor([1.0, 1.0, 1.0, 1.0, 1.0, 1.0], device=DEV), ref=None)
    train = binding.Train(max_seqs=1, device=DEV)
    got = run_policy(train, c, per_token=True)
    assert got["d"][0] == 0 and got["d"][1] == 0 and got["d"][3] == 0 and torch.isfinite(got["d"]).all() and torch.isfinite(got["stats"][0])
    for x in (0.0, 1e-20, 1e-7, 3e-4, 0.1, 0.4999, 0.5001, -0.4999, -0.5001, 3.0, -8.0, -100.0):
        lp = torch.full((n,), -1.0, device=DEV)
        c = dict(c, lp=lp, old=lp.clone(), ref=(lp.double() + x).float())
        kw = dict(kl=1.0, per_token=True)
        check_policy(c, run_policy(train, c, **kw), **kw)


def test_policy_gradient_against_differences():
    lengths = [40, 3, 25]
    train = binding.Train(max_seqs=3, device=DEV)
    for reduce in ("tokens", "sequences"):
        c = policy_case(lengths, masked=0.2, seed=3)
        on = c["t"] >= 0
        for name in ("lp", "old", "ref"):
            c[name] = torch.where(on, c[name], 0.0)
        c["lp"] = c["lp"].float()
        got = run_policy(train, c, kl=0.1, reduce=reduce)
        f = lambda lp: float(policy_reference(dict(c, lp=lp), 0.2, 0.28, 0.1, reduce, 1.0, False)["stats"][0])
        # away from the borders, where the loss has no derivative
        dist = torch.minimum(((c["lp"] - c["old"]).double() - math.log(0.8)).abs(), ((c["lp"] - c["old"]).double() - math.log1p(0.28)).abs())
        v = torch.where((dist > 1e-3) & on, torch.randn(c["lp"].shape, generator=gen(1), device=DEV, dtype=torch.float64), 0.0)
        h = 1e-5
        num = (f(c["lp"].double() + h * v) - f(c["lp"].double() - h * v)) / (2 * h)
        along = float((got["d"].double() * v).sum())
        assert abs(num - along) <= 1e-6 * (1 + abs(along))


def test_policy_gradient_in_place_and_left_out():
    c = policy_case([300, 20])
    train = binding.Train(max_seqs=2, device=DEV)
    got = run_policy(train, c, kl=0.02)
    lp, stats = c["lp"].clone(), torch.empty(6, device=DEV)
    assert binding.mars_policy_loss(train, lp, c["old"], c["adv"], c["t"], c["off"], stats, lp, ref_logprobs=c["ref"], clip_high=0.28, kl_coef=0.02) == 0
    assert torch.equal(lp, got["d"]) and torch.equal(stats, got["stats"])
    stats.fill_(7)
    assert binding.mars_policy_loss(train, c["lp"], c["old"], c["adv"], c["t"], c["off"], stats, ref_logprobs=c["ref"], clip_high=0.28, kl_coef=0.02) == 0
    assert torch.equal(stats, got["stats"])


def test_offsets_that_pass_the_tokens_or_decrease_touch_nothing_else():
    """Bad offsets give unspecified shares, never an access outside the arrays; the next call is right again."""
    c = policy_case([50, 60, 70])
    train = binding.Train(max_seqs=3, device=DEV)
    good = run_policy(train, c)
    for off in ([0, 50, 110, 5000], [-7, 50, 110, 180], [100, 20, 170, 30], [180, 180, 180, 180]):
        bad = dict(c, off=torch.tensor(off, dtype=torch.int32, device=DEV))
        got = run_policy(train, bad)
        if off[0] <= off[1] <= off[2] <= off[3]:
            check_policy(bad, got)
        again = run_policy(train, c)
        assert torch.equal(again["d"], good["d"]) and torch.equal(again["stats"], good["stats"])


# -------------------------------------------------------------------------- streams, graphs, large offsets

def all_calls(seed=0):
    """One call of every operator on a handle: a function that makes it and a list of its outputs."""
    train = binding.Train(max_width=520, max_experts=130, max_seqs=7, device=DEV)
    rope = binding.Rope(64, device=DEV)
    c = norm_case(LAYER, (300, 520), B, B, B, seed=seed, add=True, bias=True)
    y, s, dx = (torch.empty(300, 520, device=DEV, dtype=B) for _ in range(3))
    rstd, mean, dw, db = torch.empty(300, device=DEV), torch.empty(300, device=DEV), torch.empty(520, device=DEV), torch.empty(520, device=DEV)
    q = normal(gen(seed), 300, 8, 64, dtype=B)
    pos, oq = torch.arange(300, device=DEV, dtype=torch.int32) * 7, torch.empty_like(q)
    z = router_logits(300, 130, F, seed=seed)
    r = dict(idx=torch.empty(300, 5, device=DEV, dtype=torch.int32), w=torch.empty(300, 5, device=DEV), lse=torch.empty(300, device=DEV),
             counts=torch.empty(130, device=DEV, dtype=torch.int32), off=torch.empty(131, device=DEV, dtype=torch.int32),
             sums=torch.empty(130, device=DEV), losses=torch.empty(2, device=DEV))
    dz, dwt = torch.empty_like(z), normal(gen(seed + 1), 300, 5)
    p = policy_case([1000, 0, 40, 2000, 7, 900, 53], seed=seed)
    stats, d = torch.empty(6, device=DEV), torch.empty_like(p["lp"])

    def go(stream=None):
        st = [binding.mars_norm(train, LAYER, c["x"], c["w"], EPS, y, rstd=rstd, mean=mean, bias=c["b"], add=c["add"], out_sum=s, stream=stream),
              binding.mars_norm_grad(train, LAYER, c["dy"], s, c["w"], rstd, dx, dw, mean=mean, db=db, d_sum=c["d_sum"], stream=stream),
              binding.mars_rope(rope, pos, q, oq, stream=stream),
              binding.mars_router(train, z, r["idx"], r["w"], r["lse"], r["counts"], r["off"], r["sums"], r["losses"], stream=stream),
              binding.mars_router_grad(train, z, r["idx"], r["lse"], r["counts"], dz, d_weights=dwt, balance_coef=0.1, z_coef=0.1, stream=stream),
              binding.mars_policy_loss(train, p["lp"], p["old"], p["adv"], p["t"], p["off"], stats, d, ref_logprobs=p["ref"], kl_coef=0.1,
                                       reduce="sequences", stream=stream)]
        assert st == [0] * 6, st

    outs = [y, s, dx, rstd, mean, dw, db, oq, dz, stats, d] + list(r.values())
    inputs = dict(c=c, q=q, z=z, p=p, train=train)
    return go, outs, inputs


def test_same_bits_every_time_on_another_stream_and_in_a_graph():
    go, outs, inputs = all_calls()
    go()
    want = [t.clone() for t in outs]

    def same():
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
            a.zero_()
        torch.cuda.synchronize()

    for _ in range(5):
        go()
        same()
    side = torch.cuda.Stream()
    go(stream=side)
    same()
    with torch.cuda.stream(side):
        go()
    same()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    for _ in range(3):
        g.replay()
        same()
    # the graph reads what its inputs hold when it is replayed
    inputs["z"].copy_(router_logits(300, 130, F, seed=77))
    inputs["p"]["t"][::3] = -1
    inputs["p"]["off"].copy_(torch.tensor([0, 10, 1500, 1600, 1600, 3000, 3900, 4000], dtype=torch.int32, device=DEV))
    g.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in outs]
    go()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, outs)) and not torch.equal(outs[8], want[8]) and not torch.equal(outs[10], want[10])


def test_two_handles_on_two_streams_at_once():
    one, two = all_calls(1), all_calls(2)
    for go, outs, _ in (one, two):
        go()
    torch.cuda.synchronize()
    want = [[t.clone() for t in outs] for _, outs, _ in (one, two)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for (go, _, _), s in zip((one, two), streams):
            go(stream=s)
    torch.cuda.synchronize()
    for (_, outs, _), w in zip((one, two), want):
        assert all(torch.equal(a, b) for a, b in zip(outs, w))


def test_a_new_handle_is_ready_for_any_stream():
    side = torch.cuda.Stream()
    for _ in range(5):
        go, outs, _ = all_calls(3)
        go(stream=side)
        side.synchronize()
        got = [t.clone() for t in outs]
        go()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))


def test_calls_of_different_sizes_on_one_handle_in_turn():
    """What one call leaves in the workspace is nothing to the next."""
    train = binding.Train(max_width=4096, max_experts=512, max_seqs=3000, device=DEV)
    for E, n, W, lengths in ((512, 900, 64, [1] * 3000), (8, 20000, 4096, [70000, 3]), (128, 1, 1000, [5]), (512, 3, 8, [9] * 100)):
        z = router_logits(n, E, F, seed=E)
        got = run_router(train, z, 4)
        check_router(z, 4, got)
        c = norm_case(RMS, (n, W), B, B, B, seed=E)
        rstd = norm_reference(RMS, c["x"], c["w"], None)["rstd"].float()
        check_norm_grad(c, run_norm_grad(train, c, c["x"], rstd, None), c["x"], rstd, None, 0)
        p = policy_case(lengths, seed=n)
        check_policy(p, run_policy(train, p, reduce="sequences"), reduce="sequences")


def test_rows_beyond_32_bit_offsets():
    """Row strides that put the last rows more than 2^31 elements from the first."""
    n, ld = 70001, 31744
    buf = torch.empty(n, ld, dtype=B, device=DEV)
    W, g = 64, gen(1)
    parts = [buf[:, 1000 * i:1000 * i + W] for i in range(6)]      # x, dy, y, dx, logits, d_logits
    for p in (parts[0], parts[1], parts[4]):
        p.copy_(normal(g, n, W, dtype=B))
    w = normal(g, W, mean=1.0, dtype=B)
    train = binding.Train(max_width=W, max_experts=W, device=DEV)
    rstd, dw = torch.empty(n, device=DEV), torch.empty(W, device=DEV)
    assert binding.mars_norm(train, RMS, parts[0], w, EPS, parts[2], rstd=rstd) == 0
    assert binding.mars_norm_grad(train, RMS, parts[1], parts[0], w, rstd, parts[3], dw) == 0
    x, dy = parts[0].contiguous(), parts[1].contiguous()
    ref = norm_reference(RMS, x, w, None)
    assert worst(parts[2], ref["y"], rounded(B, ref["y"], ref["tol"])) <= 1
    back = norm_grad_reference(RMS, dy, x, w, None, rstd)
    assert worst(parts[3], back["dx"], rounded(B, back["dx"], back["tol_dx"])) <= 1 and worst(dw, back["dw"], back["tol_dw"]) <= 1
    z = parts[4]
    got = run_router(train, z, 4)
    check_router(z.contiguous(), 4, got)
    dwt = normal(g, n, 4)
    assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], parts[5], d_weights=dwt, balance_coef=0.3) == 0
    want, tol = router_grad_reference(z, 4, got, dwt, True, 0.3, 0.0)
    assert worst(parts[5], want, rounded(B, want, tol)) <= 1
    rope = binding.Rope(64, device=DEV)
    pos = torch.arange(n, device=DEV, dtype=torch.int32)
    q = parts[0].unflatten(1, (1, 64))
    assert binding.mars_rope(rope, pos, q, q) == 0
    want, tol = rope_reference(x.unflatten(1, (1, 64)), pos, rope.frequencies(), 64, "half", 1.0, False)
    assert worst(q, want, tol) <= 1


# ------------------------------------------------------------------------------------ a run of them together

def test_an_update_through_norm_log_probs_and_policy_loss():
    """The last norm, the log-probs of the response, the clipped loss and its way back to the residual stream and the weights;
    each step against fp64 on what the step before it gave."""
    n, hid, voc, lengths = 300, 264, 1013, [100, 0, 120, 80]
    g = gen(21)
    x, add = normal(g, n, hid, dtype=B), normal(g, n, hid, dtype=B)
    w = normal(g, hid, std=0.1, mean=1.0, dtype=B)
    head = normal(g, voc, hid, std=0.05, dtype=B)
    targets = torch.randint(voc, (n,), generator=g, device=DEV, dtype=torch.int32)
    targets[torch.rand(n, generator=g, device=DEV) < 0.3] = -1
    off = torch.tensor([0, 100, 100, 220, 300], dtype=torch.int32, device=DEV)
    train, update = binding.Train(max_width=hid, max_seqs=4, device=DEV), binding.Update(hid, voc, n, device=DEV)
    h, s, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device=DEV)
    lp, lse, d_lp, stats = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(6, device=DEV)
    d_h, d_head, dx, dw = torch.empty_like(x), torch.empty_like(head), torch.empty_like(x), torch.empty(hid, device=DEV)
    adv = normal(g, 4)

    def go(old):
        assert binding.mars_norm(train, RMS, x, w, EPS, h, rstd=rstd, add=add, out_sum=s) == 0
        assert binding.mars_logprob(update, h, head, targets, 1.0, lp, lse) == 0
        assert binding.mars_policy_loss(train, lp, old, adv, targets, off, stats, d_lp, reduce="sequences") == 0
        assert binding.mars_logprob_grad(update, h, head, targets, 1.0, lse, d_lp, d_h, d_head, logprobs=lp) == 0
        assert binding.mars_norm_grad(train, RMS, d_h, s, w, rstd, dx, dw) == 0

    go(torch.zeros(n, device=DEV))
    old = (lp + normal(g, n, std=0.2)).clamp(max=0)
    graph = torch.cuda.CUDAGraph()
    go(old)
    plain = [t.clone() for t in (stats, d_lp, d_h, d_head, dx, dw)]
    with torch.cuda.graph(graph):
        go(old)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(plain, (stats, d_lp, d_h, d_head, dx, dw)))
    c = dict(lp=lp, old=old, t=targets, off=off, adv=adv, ref=None)
    check_policy(c, dict(stats=stats, d=d_lp), low=0.2, high=0.2, reduce="sequences")
    # in fp64 from the bf16 hidden states on: d loss / d logits, then back; d and d_hidden are rounded to bf16 on the way
    z = h.double() @ head.double().t()
    p = torch.softmax(z, 1)
    on = targets >= 0
    d = -p * d_lp.double()[:, None]
    d[torch.arange(n), targets.clamp(min=0).long()] += d_lp.double()
    d[~on] = 0
    ref = norm_grad_reference(RMS, d @ head.double(), s, w, None, rstd)
    far = lambda a, b: float((a.double() - b).norm() / b.norm())
    # two roundings to bf16 (d, d_hidden) and the result's, each 2^-8 of an entry at most, through a projection and a weight near 1
    assert far(dx, ref["dx"]) <= 4 * 2.0 ** -8 and far(dw, ref["dw"]) <= 4 * 2.0 ** -8 and far(d_head, d.t() @ h.double()) <= 3 * 2.0 ** -8
    f = lambda t: float(policy_reference(dict(c, lp=t), 0.2, 0.2, 0.0, "sequences", 1.0, False)["stats"][0])
    assert abs(f(lp) - float(stats[0])) <= 1e-5


def test_a_router_feeds_the_experts_products():
    """offsets of the router are the expert_off of the products over the rows permuted by expert."""
    n, E, k, d_in, d_out = 200, 12, 3, 64, 72
    g = gen(31)
    train, update = binding.Train(max_experts=E, device=DEV), binding.Update(device=DEV)
    x, w = normal(g, n, d_in, dtype=B), normal(g, E, d_out, d_in, std=0.1, dtype=B)
    z = router_logits(n, E, F, seed=4)
    live = torch.rand(n, generator=g, device=DEV) < 0.8
    got = run_router(train, z, k, live)
    flat = got["idx"].flatten().long()
    order = torch.sort(torch.where(flat < 0, E, flat), stable=True).indices          # padding behind the last expert
    rows = x[order // k].contiguous()
    y = torch.zeros(n * k, d_out, device=DEV)
    assert binding.mars_expert_matmul(update, rows, got["off"], w, y) == 0 and update.poll_status() == 0
    used = int(got["off"][-1])
    assert used == k * int(live.sum()) and (y[used:] == 0).all()
    want = torch.einsum("rd,rod->ro", rows[:used].double(), w.double()[flat[order[:used]]])
    # at most (64 / 16 + 16) fp32 steps of the sum of absolute products
    tol = 20 * 2.0 ** -23 * torch.einsum("rd,rod->ro", rows[:used].double().abs(), w.double().abs()[flat[order[:used]]])
    assert worst(y[:used], want, tol) <= 1
    # the gradient of sum(weights y) to the weights goes back through the router
    dw = torch.empty(n * k, device=DEV)
    dw[order] = y.sum(1)
    d = torch.empty_like(z)
    assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], d, d_weights=dw.view(n, k), balance_coef=0.01) == 0
    ref, tol = router_grad_reference(z, k, got, dw.view(n, k), True, 0.01, 0.0)
    assert worst(d, ref, rounded(F, ref, tol)) <= 1


def test_handles_refuse_what_they_were_not_made_for():
    train = binding.Train(max_width=64, device=DEV)
    z = router_logits(4, 8, F)
    assert binding.mars_router(train, z, torch.empty(4, 2, device=DEV, dtype=torch.int32), torch.empty(4, 2, device=DEV)) == 1
    x, w = torch.zeros(4, 72, device=DEV), torch.zeros(72, device=DEV)
    assert binding.mars_norm(train, RMS, x, w, EPS, torch.empty_like(x)) == 1
    c = policy_case([3])
    assert binding.mars_policy_loss(train, c["lp"], c["old"], c["adv"], c["t"], c["off"], torch.empty(6, device=DEV)) == 1
    with pytest.raises(binding.MarsError):
        binding.Train(device=DEV)
    with pytest.raises(binding.MarsError):
        binding.Rope(3, device=DEV)
    rope = binding.Rope(64, device=DEV)
    q = torch.zeros(4, 1, 32, device=DEV)
    assert binding.mars_rope(rope, torch.zeros(4, device=DEV, dtype=torch.int32), q, q) == 1


# ------------------------------------------------------------------------- what the tests above leave out

@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
def test_far_angles_against_frequencies_of_60_digits(scaling):
    """Neither the frequencies nor the turns of the library: both from theta, the exponent and the scaling."""
    rotary, half = 96, 48
    rope = binding.Rope(rotary, theta=5e5, scaling=scaling, factor=8.0, trained_positions=32768, device=DEV)
    positions = [0, 1, -1, 40_000, 131_071, 1_000_003, 2 ** 31 - 1, -2 ** 31]
    x = torch.zeros(len(positions), 1, rotary, device=DEV)
    x[..., :half] = 1                                            # (1, 0) turns to (cos, sin)
    out = torch.empty_like(x)
    assert binding.mars_rope(rope, torch.tensor(positions, dtype=torch.int32, device=DEV), x, out) == 0
    out = out[:, 0].cpu().tolist()
    with localcontext() as ctx:
        ctx.prec = 60
        for j, f in enumerate(exact_frequencies(rotary, ["none", "linear", "base", "parts"].index(scaling), 5e5)):
            for i, p in enumerate(positions):
                turns = p * f / TWO_PI
                angle = 2 * math.pi * float(turns - turns.to_integral_value())
                # half a step of the table's entry (2^-58 for its chain) and of the product; the fraction in fp32 and the functions 2^-22
                e = 2.0 ** -22 + 2 * math.pi * abs(float(turns)) * (2.0 ** -52 + 2.0 ** -58)
                assert abs(out[i][j] - math.cos(angle)) <= e and abs(out[i][half + j] - math.sin(angle)) <= e, (p, j)


@pytest.mark.parametrize("t", [B, H])
@pytest.mark.parametrize("width", [128, 1111, 2048, 8192])
@pytest.mark.parametrize("kind", [RMS, LAYER])
def test_weight_gradients_are_rounded_once(kind, width, t):
    """Sums next to the middle between two numbers of 16 bits: what decides is far below fp32's last bit."""
    train = binding.Train(max_width=width, device=DEV)
    n, u = 4096, U[t]                                            # the three rows that are not zeros lie in blocks of their own
    x, w, ones = torch.ones(n, width, device=DEV), torch.ones(width, device=DEV), torch.ones(n, device=DEV)
    mean = torch.zeros(n, device=DEV) if kind == LAYER else None
    for sign, parts, want in ((1, (1.0, u, 2.0 ** -40), 1 + 2 * u), (-1, (1 + 2 * u, u, -2.0 ** -40), 1 + 2 * u)):
        for accumulate in (False, True):
            dy = torch.zeros(n, width, device=DEV)
            dy[n // 2], dy[n - 1] = sign * parts[1], sign * parts[2]
            dw = torch.full((width,), sign * parts[0], device=DEV, dtype=t) if accumulate else torch.full((width,), 77.0, device=DEV, dtype=t)
            if not accumulate:
                dy[0] = sign * parts[0]
            db = dw.clone() if kind == LAYER else None
            assert binding.mars_norm_grad(train, kind, dy, x, w, ones, torch.empty_like(x), dw, mean=mean, db=db, accumulate=accumulate) == 0
            assert (dw.double() == sign * want).all() and (db is None or torch.equal(db, dw)), (dw[0], sign * want)


@pytest.mark.parametrize("E,k", [(8, 8), (64, 4), (65, 8), (128, 8), (200, 3), (512, 8)])
@pytest.mark.parametrize("t", [F, B, H])
def test_a_nan_beside_nothing_but_minus_infinity(E, k, t):
    """Neither of few nor of many rows is such a row one without logits: its weights and the sums are NaN, its choices different experts."""
    train = binding.Train(max_experts=E, device=DEV)
    for n in (70, 8200):
        for at in (0, E // 2, E - 1):
            for sign in (math.nan, -math.nan):
                z = router_logits(n, E, t, seed=1)
                want = run_router(train, z, k)
                z[n - 3] = -math.inf
                z[n - 3, at] = sign
                got = run_router(train, z, k)
                assert got["w"][n - 3].isnan().all() and got["lse"][n - 3].isnan() and got["sums"].isnan().all() and got["losses"].isnan().all()
                chosen = got["idx"][n - 3].tolist()
                assert len(set(chosen)) == k and 0 <= min(chosen) and max(chosen) < E
                assert int(got["off"][-1]) == n * k and torch.equal(got["counts"].long(), torch.bincount(got["idx"].flatten().long(), minlength=E))
                keep = torch.arange(n, device=DEV) != n - 3
                assert all(torch.equal(got[name][keep], want[name][keep]) for name in ("idx", "w", "lse"))


@pytest.mark.parametrize("lengths", [[3, 0, 1500, 600, 1], [700, 6000, 31, 0, 900]], ids=["short", "long"])
@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("reduce", ["tokens", "sequences"])
def test_policy_tensors_that_start_off_16_bytes(lengths, per_token, reduce):
    """Slices of a packed batch: the same bits as from the start of an allocation."""
    train = binding.Train(max_seqs=len(lengths), device=DEV)
    c = policy_case(lengths, per_token=per_token, seed=5, before=3, behind=2)
    want = run_policy(train, c, kl=0.04, reduce=reduce, per_token=per_token)
    check_policy(c, want, kl=0.04, reduce=reduce, per_token=per_token)

    def moved(v, by):
        buf = torch.full((v.shape[0] + by,), 3, device=DEV, dtype=v.dtype)
        buf[by:] = v
        return buf[by:]

    names = ["lp", "old", "ref", "t", "off", "adv"]
    for off_by in [{name: by} for name in names for by in (1, 2, 3)] + [dict.fromkeys(names, 1), dict(lp=1, old=2, ref=3)]:
        a = {name: moved(v, off_by[name]) if name in off_by else v for name, v in c.items()}
        assert (a["lp"].data_ptr() % 16 != 0) == ("lp" in off_by)
        stats = torch.full((7,), 77.0, device=DEV)[1:]
        for by in (0, 1, 2):
            room = torch.full((len(c["lp"]) + 4,), 77.0, device=DEV)
            d = room[by:by + len(c["lp"])]
            assert binding.mars_policy_loss(train, a["lp"], a["old"], a["adv"], a["t"], a["off"], stats, d, ref_logprobs=a["ref"], clip_low=0.2,
                                            clip_high=0.28, kl_coef=0.04, reduce=reduce, per_token=per_token) == 0
            assert torch.equal(stats, want["stats"]) and torch.equal(d, want["d"])
            assert (room[:by] == 77).all() and (room[by + len(d):] == 77).all()


@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("xt,yt,wt", [(B, B, B), (F, B, F), (F, F, B), (H, H, F)])
def test_norm_weights_that_start_off_16_bytes(kind, xt, yt, wt):
    """Rows in whole 16-byte pieces, weight and bias not."""
    train = binding.Train(max_width=2048, device=DEV)
    for shape in ((300, 256), (70, 2048), (40, 6, 128)):
        c = norm_case(kind, shape, xt, yt, wt, add=True, bias=kind == LAYER)
        for names in (("w",), ("b",), ("w", "b")):
            a = dict(c)
            for name in names:
                if a[name] is not None:
                    a[name] = torch.cat([a[name].new_full((1,), math.nan), a[name]])[1:]
            got = run_norm(train, a, yt)
            check_norm(a, got, yt, 0)
            back = run_norm_grad(train, a, got["s"], got["rstd"], got["mean"])
            check_norm_grad(a, back, got["s"], got["rstd"], got["mean"], 0)


@pytest.mark.parametrize("n,E,k", [(8192, 8, 2), (20000, 60, 4), (40000, 128, 8), (12345, 384, 8), (9000, 128, 12), (5000, 600, 8)])
@pytest.mark.parametrize("t", [F, B])
def test_router_of_many_rows_gives_the_same_bits_in_every_output(n, E, k, t):
    train = binding.Train(max_experts=E, device=DEV)
    z = router_logits(n, E, t, seed=3)
    live = torch.rand(n, generator=gen(2), device=DEV) < 0.9
    want = run_router(train, z, k, live)
    assert all(torch.isfinite(v).all() for v in want.values())
    for _ in range(12):
        got = run_router(train, z, k, live)
        assert all(torch.equal(got[name], want[name]) for name in want)


@pytest.mark.parametrize("E,k,t", [(20, 3, F), (61, 5, F), (128, 8, F), (128, 8, B), (384, 6, F), (600, 4, F)])
@pytest.mark.parametrize("renormalise", [True, False])
def test_router_gradient_of_logits_far_from_zero(E, k, t, renormalise):
    """A common offset changes no probability: lse is rounded to its own last bit, the gradient is not to inherit that."""
    for n, middle, std in ((70, 1000.0, 1.0), (9000, -4096.0, 1.0), (300, 3e5, 1.0), (500, 0.0, 16.0), (40, 1e7, 0.0)):
        train = binding.Train(max_experts=E, device=DEV)
        z = (router_logits(n, E, F, seed=4, std=1.0) * std + middle).to(t)
        got = run_router(train, z, k, renormalise=renormalise)
        dw = normal(gen(5), n, k, mean=0.5)
        d = torch.empty_like(z)
        cb, cz = 0.01 * n, 1e-3 * n / max(1.0, abs(middle))
        assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], d, d_weights=dw, balance_coef=cb, z_coef=cz,
                                        renormalise=renormalise) == 0
        # the reference that takes lse as it is given, with the exact one in its place
        exact = dict(got, lse=torch.logsumexp(z.double(), 1))
        want, tol = router_grad_reference(z, k, exact, dw, renormalise, cb, cz)
        # exponentials below the normal numbers are 0: 2^-126 times what multiplies them, |dw| <= 6 and as much of the losses
        assert worst(d, want, rounded(t, want, tol) + 12 * 2.0 ** -126) <= 1, (n, middle, std)


@pytest.mark.parametrize("E,k,t", [(16, 6, F), (61, 5, B), (128, 8, F), (128, 8, H), (600, 4, B)])
@pytest.mark.parametrize("renormalise", [True, False])
def test_router_gradient_of_rows_at_the_lowest_number(E, k, t, renormalise):
    """All logits alike, whatever they are: every expert has a probability of 1 / E."""
    train = binding.Train(max_experts=E, device=DEV)
    n = 50
    z = router_logits(n, E, t, seed=6)
    z[7:20] = torch.finfo(t).min
    got = run_router(train, z, k, renormalise=renormalise)
    dw = normal(gen(5), n, k, mean=0.5)
    d = torch.empty_like(z)
    assert binding.mars_router_grad(train, z, got["idx"], got["lse"], got["counts"], d, d_weights=dw, balance_coef=0.5, renormalise=renormalise) == 0
    same = z.clone()
    same[7:20] = 0.0                                             # the same rows by another offset: lse = log E
    want, tol = router_grad_reference(same, k, dict(got, lse=torch.logsumexp(same.double(), 1)), dw, renormalise, 0.5, 0.0)
    assert worst(d, want, rounded(t, want, tol)) <= 1
