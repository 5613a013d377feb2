"""Operators of a training pass, host side (no device): sizes, refusals that are decided before any CUDA call, the
rotation's frequencies and the binding's checks of tensors."""
import ctypes
import math
from decimal import Decimal

import pytest
import torch

from helpers import exact_frequencies
from paper_2511_11373_b200 import binding

A = 1 << 20                                              # a made-up address, aligned to everything


@pytest.fixture(scope="module")
def lib():
    from paper_2511_11373_b200 import build
    build.build()
    return binding.lib()


@pytest.mark.parametrize("w,e,s", [(1, 0, 0), (2048, 0, 0), (8192, 0, 0), (0, 1, 0), (0, 1024, 0), (0, 0, 1), (0, 0, 1 << 20),
                                   (2048, 128, 1024)])
def test_workspace_sizes(lib, w, e, s):
    b = lib.mars_train_workspace_bytes(w, e, s)
    assert b > 0 and b % 256 == 0
    # per-block sums of the widest row or of the experts, and counters
    assert b <= 8192 + 2 * 148 * 4 * (3 * min(w, 256) + 2 * w) + 148 * 2 * (4 * e + 8) + 4 * e + 4 * s + 148 * 8 * 32 * bool(s)


@pytest.mark.parametrize("w,e,s", [(0, 0, 0), (-1, 0, 0), (8193, 0, 0), (0, 1025, 0), (0, -1, 0), (0, 0, (1 << 20) + 1), (8, 8, -1)])
def test_sizes_that_are_not_supported(lib, w, e, s):
    assert lib.mars_train_workspace_bytes(w, e, s) == 0
    out = ctypes.c_void_p()
    assert lib.mars_train_create(w, e, s, ctypes.c_void_p(256), 1 << 40, ctypes.byref(out)) == 2 and not out.value


def test_bad_workspaces_and_null_handles(lib):
    out = ctypes.c_void_p()
    assert lib.mars_train_create(8, 0, 0, None, 1 << 30, ctypes.byref(out)) == 1
    assert lib.mars_train_create(8, 0, 0, ctypes.c_void_p(128), 1 << 30, ctypes.byref(out)) == 1
    assert lib.mars_train_create(8, 0, 0, ctypes.c_void_p(256), 256, ctypes.byref(out)) == 1
    assert lib.mars_train_create(8, 0, 0, ctypes.c_void_p(256), 1 << 30, None) == 1
    assert lib.mars_train_free(None) == 6 and lib.mars_rope_free(None) == 6
    norm, policy = binding.mars_norm_t(0, 8, 1, 1, 1, 1, 1e-6, 0), binding.mars_policy_t(0.2, 0.2, 0, 1, 0, 0)
    assert lib.mars_norm(None, None, ctypes.byref(norm), 1, A, 8, None, 0, None, 0, A, None, A, 8, None, None) == 6
    assert lib.mars_norm_grad(None, None, ctypes.byref(norm), 1, A, 8, A, 8, A, None, A, None, 0, A, 8, None, None, 0, 0) == 6
    assert lib.mars_rope(None, None, 1, A, 8, 1, A, 8, 1, A, 8, None, 0, 0, None, 0, 0) == 6
    assert lib.mars_router(None, None, 1, 8, 2, A, 8, 0, None, 1, A, A, None, None, None, None, None) == 6
    assert lib.mars_router_grad(None, None, 1, 8, 2, A, 8, 0, A, A, A, None, 1, 0.0, 0.0, A, 8) == 6
    assert lib.mars_policy_loss(None, None, ctypes.byref(policy), 1, 1, A, A, A, A, None, A, A, A) == 6


# The checks of the calls, through a made-up handle (device, SMs, largest sizes, ...).  What they let pass ends here in a CUDA error,
# since there is no device; with one these calls could reach it, so they are not made.
no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")


def fake(*fields):
    h = (ctypes.c_int64 * 32)()
    ctypes.memmove(h, (ctypes.c_int32 * len(fields))(*fields), 4 * len(fields))
    for i in range(3, 32):
        h[i] = A << 8
    return ctypes.cast(h, ctypes.c_void_p), h


@no_device
def test_refusals_of_norms(lib):
    handle, keep = fake(0, 148, 64, 0, 0)
    F, B, H = 0, 1, 2

    def fwd(kind=0, width=64, heads=1, xt=B, yt=B, wt=B, eps=1e-6, n=4, x=A, ldx=64, add=None, lda=64, s=None, lds=64, w=A + 65536,
            b=None, y=A + 8192, ldy=64, mean=None, rstd=None):
        form = binding.mars_norm_t(kind, width, heads, xt, yt, wt, eps, 0)
        return lib.mars_norm(handle, None, ctypes.byref(form), n, x, ldx, add, lda, s, lds, w, b, y, ldy, mean, rstd)

    assert fwd() == 3 and fwd(y=A) == 3 and fwd(kind=1, b=A + 70000, mean=A + 80000, rstd=A + 90000) == 3 and fwd(n=0, x=None, y=None) == 0
    assert fwd(add=A + 16384, s=A) == 3 and fwd(xt=F, yt=B) == 3 and fwd(xt=F, yt=H) == 3 and fwd(width=7, ldx=7, ldy=9) == 3
    assert fwd(heads=2, width=32) == 3 and fwd(x=A, ldx=128, y=A + 128, ldy=128) == 3
    for bad in (dict(kind=2), dict(kind=-1), dict(width=0), dict(width=65, ldx=65, ldy=65), dict(heads=0), dict(xt=3), dict(yt=-1), dict(wt=7),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan), dict(n=-1), dict(x=None), dict(y=None), dict(w=None),
                dict(ldx=63), dict(ldy=63), dict(ldx=1 << 40), dict(x=A + 1), dict(y=A + 8193), dict(w=A + 65537),
                dict(heads=2, width=64, ldx=127, ldy=128), dict(n=2 ** 30, heads=4, width=8),
                dict(s=A + 16384), dict(add=A + 16384, lda=60), dict(mean=A + 80000), dict(b=A + 70000), dict(rstd=A + 90001),
                dict(y=A + 64), dict(y=A, ldy=80, n=3), dict(add=A + 16384, s=A, y=A), dict(add=A + 16384, s=A + 16, y=A + 8192),
                dict(rstd=A + 8192), dict(rstd=A), dict(w=A + 8192), dict(kind=1, mean=A + 80000, rstd=A + 80004)):
        assert fwd(**bad) == 1, bad
    assert fwd(xt=B, yt=F) == 2 and fwd(xt=B, yt=H) == 2
    form = None
    assert lib.mars_norm(handle, None, form, 1, A, 64, None, 0, None, 0, A, None, A, 64, None, None) == 1

    def back(kind=0, n=4, dy=A, lddy=64, x=A + 8192, ldx=64, w=A + 65536, mean=None, rstd=A + 80000, ds=None, ldds=64, dx=A + 16384, lddx=64,
             dw=A + 90112, db=None, dwt=F):
        f = binding.mars_norm_t(kind, 64, 1, B, B, B, 1e-6, 0)
        return lib.mars_norm_grad(handle, None, ctypes.byref(f), n, dy, lddy, x, ldx, w, mean, rstd, ds, ldds, dx, lddx, dw, db, dwt, 0)

    assert back() == 3 and back(dw=None) == 3 and back(dx=A) == 3 and back(dx=A + 8192) == 3 and back(ds=A + 32768, dx=A + 32768) == 3
    assert back(kind=1, mean=A + 70000, db=A + 95000) == 3 and back(n=0, dy=None, x=None, dx=None, rstd=None) == 3
    for bad in (dict(rstd=None), dict(kind=1), dict(mean=A + 70000), dict(db=A + 95000), dict(dwt=3), dict(dw=A + 90114), dict(dx=None), dict(dy=None),
                dict(x=None), dict(w=None), dict(dx=A + 64), dict(dx=A + 8192, lddx=72), dict(dw=A), dict(dw=A + 16384), dict(dw=A + 80000),
                dict(kind=1, mean=A + 70000, db=A + 90112), dict(ds=A + 32768, ldds=8), dict(dx=A + 80000 - 64)):
        assert back(**bad) == 1, bad


@no_device
def test_refusals_of_the_router(lib):
    handle, keep = fake(0, 148, 0, 64, 0)

    def fwd(rows=4, E=64, k=8, z=A, ld=64, t=0, live=None, idx=A + 8192, w=A + 16384, lse=None, counts=None, off=None, sums=None, losses=None):
        return lib.mars_router(handle, None, rows, E, k, z, ld, t, live, 1, idx, w, lse, counts, off, sums, losses)

    assert fwd() == 3 and fwd(rows=0, z=None, idx=None, w=None) == 3 and fwd(E=7, ld=9, k=7, t=2) == 3 and fwd(live=A + 40001) == 3
    for bad in (dict(E=65, ld=65), dict(E=0), dict(k=0), dict(k=33), dict(E=4, k=5), dict(rows=-1), dict(z=None), dict(ld=63), dict(t=3), dict(z=A + 2),
                dict(idx=None), dict(w=None), dict(idx=A + 8193), dict(idx=A), dict(w=A + 8192), dict(lse=A + 8196), dict(counts=A + 4),
                dict(losses=A + 3), dict(off=A + 24576, counts=A + 24576 + 256), dict(live=A + 8192), dict(rows=1 << 29, k=8)):
        assert fwd(**bad) == 1, bad

    def back(rows=4, E=64, k=8, z=A, ld=64, t=0, idx=A + 8192, lse=A + 16384, counts=A + 20480, dw=None, b=0.1, c=0.1, d=A + 32768, ldd=64):
        return lib.mars_router_grad(handle, None, rows, E, k, z, ld, t, idx, lse, counts, dw, 1, b, c, d, ldd)

    assert back() == 3 and back(d=A) == 3 and back(rows=0, z=None, idx=None, lse=None, counts=None, d=None) == 0
    for bad in (dict(idx=None), dict(lse=None), dict(counts=None), dict(d=None), dict(d=A, ldd=72), dict(d=A + 256), dict(ldd=60), dict(b=math.inf),
                dict(c=math.nan), dict(d=A + 8192), dict(dw=A + 32768), dict(k=33), dict(E=65), dict(d=A + 32770)):
        assert back(**bad) == 1, bad


@no_device
def test_refusals_of_the_policy_loss(lib):
    handle, keep = fake(0, 148, 0, 0, 16)

    def call(n=4, seqs=2, off=A, t=A + 4096, lp=A + 8192, old=A + 12288, ref=None, adv=A + 16384, stats=A + 20480, d=A + 24576, low=0.2, high=0.2,
             kl=0.0, scale=1.0, reduce=0, per=0):
        f = binding.mars_policy_t(low, high, kl, scale, reduce, per)
        return lib.mars_policy_loss(handle, None, ctypes.byref(f), n, seqs, off, t, lp, old, ref, adv, stats, d)

    assert call() == 3 and call(d=None) == 3 and call(d=A + 8192) == 3 and call(n=0, t=None, lp=None, old=None, d=None) == 3
    assert call(low=1.0, high=0.0) == 3 and call(ref=A + 28672, kl=0.1) == 3 and call(n=0, t=None, lp=None, old=None, d=None, adv=None, per=1) == 3
    for bad in (dict(n=-1), dict(n=(1 << 30) + 1), dict(seqs=0), dict(seqs=17), dict(low=-0.1), dict(low=1.5), dict(high=-0.1), dict(high=math.inf),
                dict(high=math.nan), dict(low=math.nan), dict(kl=0.1), dict(kl=math.inf, ref=A + 28672), dict(scale=math.nan), dict(reduce=3),
                dict(reduce=-1), dict(off=None), dict(stats=None), dict(t=None), dict(lp=None), dict(old=None), dict(adv=None), dict(lp=A + 8193),
                dict(d=A + 8196), dict(d=A + 12288), dict(stats=A + 8192), dict(d=A + 20484), dict(d=A), dict(ref=A + 24576), dict(adv=A + 24576),
                dict(stats=A + 4)):
        assert call(**bad) == 1, bad
    assert lib.mars_policy_loss(handle, None, None, 1, 1, A, A, A, A, None, A, A, A) == 1


def rope_form(rotary=64, layout=0, scaling=0, theta=1e4, factor=4.0, trained=4096.0, fast=32.0, slow=1.0, scale=1.0):
    return binding.mars_rope_form_t(rotary, layout, scaling, 0, theta, factor, trained, fast, slow, scale)


@pytest.mark.parametrize("bad", [dict(rotary=0), dict(rotary=1), dict(rotary=3), dict(rotary=514), dict(layout=2), dict(layout=-1), dict(scaling=4),
                                 dict(theta=0.0), dict(theta=math.inf), dict(scale=0.0), dict(scale=1e39), dict(scaling=1, factor=0.0),
                                 dict(scaling=2, rotary=2), dict(scaling=3, trained=0.0), dict(scaling=3, fast=1.0), dict(scaling=3, slow=-1.0),
                                 dict(scaling=3, fast=math.inf), dict(scaling=1, factor=math.nan)])
def test_rotations_that_are_refused(lib, bad):
    f, out, table = rope_form(**bad), ctypes.c_void_p(), (ctypes.c_double * 512)()
    assert lib.mars_rope_bytes(ctypes.byref(f)) == 0 and lib.mars_rope_frequencies(ctypes.byref(f), table) == 1
    assert lib.mars_rope_create(ctypes.byref(f), ctypes.c_void_p(256), 1 << 20, ctypes.byref(out)) == 1 and not out.value
    with pytest.raises(ValueError):
        binding.Rope(64, layout="third")


@no_device
def test_refusals_of_the_rotation(lib):
    handle, keep = fake(0, 148, 64, 0, 0)                  # device, SMs, rotary, interleaved, scale

    def call(n=4, pos=A, dim=128, t=1, q=A + 8192, ldq=1024, hq=4, oq=A + 65536, ldoq=1024, k=A + 8192 + 1024, ldk=1024, hk=1, ok=A + 65536 + 1024,
             ldok=1024):
        return lib.mars_rope(handle, None, n, pos, dim, t, q, ldq, hq, oq, ldoq, k, ldk, hk, ok, ldok, 0)

    assert call() == 3 and call(oq=A + 8192, ok=A + 8192 + 1024) == 3 and call(hk=0, k=None, ok=None) == 3
    assert call(n=0, pos=None, q=None, oq=None, k=None, ok=None) == 0
    for bad in (dict(n=-1), dict(pos=None), dict(pos=A + 2), dict(dim=32), dict(dim=513), dict(t=3), dict(hq=0), dict(hk=-1), dict(q=None), dict(oq=None),
                dict(k=None), dict(ok=None), dict(ldq=511), dict(ldk=127), dict(oq=A + 8192 + 16), dict(oq=A + 8192, ldoq=1032),
                dict(oq=A + 8192 + 1024), dict(ok=A + 65536 + 16), dict(pos=A + 65536), dict(ok=A + 8192), dict(hq=1 << 17, ldq=1 << 25)):
        assert call(**bad) == 1, bad


@pytest.mark.parametrize("rotary", [2, 4, 64, 96, 128, 512])
@pytest.mark.parametrize("scaling", [0, 1, 2, 3])
def test_frequencies(lib, rotary, scaling):
    if scaling == 2 and rotary == 2:
        return
    f = rope_form(rotary=rotary, scaling=scaling, theta=1e6, factor=8.0, trained=32768.0, fast=32.0, slow=1.0)
    got = binding.rope_frequencies(f)
    for i in range(rotary // 2):
        theta = 1e6 * 8.0 ** (rotary / (rotary - 2)) if scaling == 2 else 1e6
        want = theta ** (-2 * i / rotary)
        if scaling == 1:
            want /= 8
        if scaling == 3:
            turns = 32768 * want / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1) / 31))
            want = keep * want + (1 - keep) * want / 8
        # pow and a handful of products in fp64: some 2^-50
        assert abs(float(got[i]) - want) <= 2.0 ** -48 * want
    if scaling == 3 and rotary == 128:
        plain = binding.rope_frequencies(rope_form(rotary=128, theta=1e6))
        assert got[0] == plain[0] and abs(float(got[-1] / plain[-1]) - 1 / 8) < 1e-12


class Fake:                                               # stands for a handle: the checks come before the library
    handle, device, max_width, max_experts, max_seqs, _forms, _index = None, torch.device("cpu"), 64, 64, 64, {}, -1

    def _stream(self, stream):
        return 0


def test_the_binding_refuses_tensors_of_another_kind():
    f, bf, z = Fake(), torch.bfloat16, torch.zeros
    x, w = z(4, 8, dtype=bf), z(8, dtype=bf)
    norm = dict(x=x, weight=w, y=z(4, 8, dtype=bf))
    for bad in (dict(x=z(8)), dict(x=z(4, 8, dtype=torch.float64)), dict(y=z(4, 9, dtype=bf)), dict(y=z(8, 4, dtype=bf).t()), dict(weight=z(9)),
                dict(rstd=z(5)), dict(rstd=z(4, dtype=bf)), dict(mean=z(4, 1)), dict(add=z(4, 8)), dict(out_sum=z(4, 8)), dict(bias=z(8)),
                dict(x=x[:, None].expand(4, 2, 8), y=z(4, 2, 8, dtype=bf)), dict(x=z(4, 2, 16, dtype=bf)[..., ::2], y=z(4, 2, 8, dtype=bf)),
                dict(y=z(1, 8, dtype=bf).expand(4, 8))):
        a = dict(norm, **bad)
        with pytest.raises(ValueError):
            binding.mars_norm(f, 0, a.pop("x"), a.pop("weight"), 1e-6, a.pop("y"), **a)
    for bad in (dict(dx=z(4, 8)), dict(dw=z(9)), dict(d_sum=z(4, 8)), dict(rstd=None), dict(db=z(8, dtype=bf)), dict(dy=z(3, 8, dtype=bf))):
        a = dict(dict(dy=x, rstd=z(4), dx=x, dw=z(8)), **bad)
        with pytest.raises(ValueError):
            binding.mars_norm_grad(f, 0, a.pop("dy"), x, w, a.pop("rstd"), a.pop("dx"), a.pop("dw"), **a)
    q, pos = z(4, 2, 8, dtype=bf), z(4, dtype=torch.int32)
    for args in ((pos.long(), q, q), (pos[:3], q, q), (pos, q[0], q[0]), (pos, q, q.float()), (pos, q, q, q, None), (pos, q, q, q[:3], q[:3]),
                 (pos, q.double(), q.double()), (pos, q.transpose(0, 1), q.transpose(0, 1))):
        with pytest.raises(ValueError):
            binding.mars_rope(f, *args)
    logits, idx, wt = z(4, 8), z(4, 2, dtype=torch.int32), z(4, 2)
    for args, kw in (((logits.double(), idx, wt), {}), ((logits, idx.long(), wt), {}), ((logits, idx, wt[:, :1]), {}), ((logits, idx[0], wt), {}),
                     ((logits, idx, wt), dict(out_offsets=z(8, dtype=torch.int32))), ((logits, idx, wt), dict(live=z(4))),
                     ((logits, idx, wt), dict(out_losses=z(1))), ((logits.t(), idx, wt), {})):
        with pytest.raises(ValueError):
            binding.mars_router(f, *args, **kw)
    with pytest.raises(ValueError):
        binding.mars_router_grad(f, logits, idx, z(4), z(8, dtype=torch.int32), logits.bfloat16())
    lp, off = z(4), z(3, dtype=torch.int32)
    ok = dict(lp=lp, old=lp, adv=z(2), t=z(4, dtype=torch.int32), off=off, stats=z(6))
    for bad, kw in ((dict(lp=z(4, dtype=bf)), {}), (dict(old=z(5)), {}), (dict(adv=z(4)), {}), (dict(adv=z(2)), dict(per_token=True)),
                    (dict(t=z(4)), {}), (dict(stats=z(5)), {}), (dict(off=off.long()), {}), ({}, dict(ref_logprobs=z(3))),
                    ({}, dict(out_d_logprobs=z(4, 1))), ({}, dict(reduce="mean"))):
        a = dict(ok, **bad)
        with pytest.raises(ValueError):
            binding.mars_policy_loss(f, a["lp"], a["old"], a["adv"], a["t"], a["off"], a["stats"], **kw)


class Passed:                                             # stands for the library: what a call passes on
    def __init__(self):
        self.forms = []

    def __getattr__(self, name):
        def call(handle, stream, form, *rest):
            self.forms.append({n: getattr(form._obj, n) for n, _ in form._obj._fields_})
            return 0
        return call


@pytest.mark.parametrize("name", ["clip_low", "clip_high", "kl_coef", "scale"])
def test_a_coefficient_that_changes_in_place_is_read_again(monkeypatch, name):
    passed, f, z = Passed(), Fake(), torch.zeros
    f._forms = {}
    monkeypatch.setattr(binding, "lib", lambda: passed)
    coef, lp = torch.tensor(0.25, dtype=torch.float64), z(4)
    args = (lp, lp, z(2), z(4, dtype=torch.int32), z(3, dtype=torch.int32), z(6))
    for value in (0.25, 0.5, 0.5, 0.125):
        coef.fill_(value)
        assert binding.mars_policy_loss(f, *args, ref_logprobs=lp, **{name: coef}) == 0
        assert passed.forms[-1][name] == value
    assert binding.mars_policy_loss(f, *args, ref_logprobs=lp, **{name: 0.125}) == 0
    assert passed.forms[-1] == passed.forms[-2] and len(f._forms) == 3          # a number and a tensor of its value are one form


def test_an_epsilon_that_changes_in_place_is_read_again(monkeypatch):
    passed, f, z = Passed(), Fake(), torch.zeros
    f._forms = {}
    monkeypatch.setattr(binding, "lib", lambda: passed)
    eps = torch.tensor(0.25)
    for value in (0.25, 0.5, 0.125):
        eps.fill_(value)
        assert binding.mars_norm(f, 0, z(4, 8), z(8), eps, z(4, 8)) == 0
        assert passed.forms[-1]["eps"] == value


@pytest.mark.parametrize("wrong", [None, [0.0, 0.0, 0.0, 0.0], 1.5, torch.tensor(0.0), torch.tensor(0, dtype=torch.int32)], ids=["none", "list", "number", "fp32", "int32"])
def test_arguments_that_are_no_tensors_of_a_call(wrong):
    """Whatever stands in a tensor's place, the refusal is the same."""
    f, z = Fake(), torch.zeros
    lp, i32 = z(4), torch.int32
    calls = [(binding.mars_policy_loss, [f, lp, lp, z(2), z(4, dtype=i32), z(3, dtype=i32), z(6)], range(1, 7)),
             (binding.mars_norm, [f, 0, z(4, 8), z(8), 1e-6, z(4, 8)], (2, 3, 5)),
             (binding.mars_norm_grad, [f, 0, z(4, 8), z(4, 8), z(8), z(4), z(4, 8)], (2, 3, 4, 5, 6)),
             (binding.mars_rope, [f, z(4, dtype=i32), z(4, 2, 8), z(4, 2, 8)], (1, 2, 3)),
             (binding.mars_router, [f, z(4, 8), z(4, 2, dtype=i32), z(4, 2)], (1, 2, 3)),
             (binding.mars_router_grad, [f, z(4, 8), z(4, 2, dtype=i32), z(4), z(8, dtype=i32), z(4, 8)], range(1, 6))]
    for call, args, places in calls:
        for at in places:
            with pytest.raises(ValueError):
                call(*args[:at], wrong, *args[at + 1:])


@pytest.mark.parametrize("rotary", [2, 80, 96, 128, 510])
@pytest.mark.parametrize("scaling", [0, 1, 2, 3])
@pytest.mark.parametrize("theta", [1e4, 1e6, 5e5])
def test_frequencies_are_rounded_once(lib, rotary, scaling, theta):
    if scaling == 2 and rotary == 2:
        return
    got = binding.rope_frequencies(rope_form(rotary=rotary, scaling=scaling, theta=theta, factor=8.0, trained=32768.0))
    for g, want in zip(got.tolist(), exact_frequencies(rotary, scaling, theta)):
        # half a step of fp64 and, in steps of 2^-64 of the value: ln theta <= 17 for the rounded exponent, the power, a product and a
        # quotient, some 24; by parts the blend has as much again from the turns, 64 in all
        assert abs(Decimal(g) - want) <= want * (Decimal(2) ** -53 + Decimal(2) ** -58)


def test_a_rotation_scaled_by_what_fp32_takes_for_zero_is_refused(lib):
    for scale, ok in ((1e-50, False), (7e-46, False), (2e-45, True), (1e-30, True)):         # fp32 goes down to 1.4e-45, halves are rounded up
        f, table = rope_form(scale=scale), (ctypes.c_double * 512)()
        assert (lib.mars_rope_bytes(ctypes.byref(f)) > 0) == ok and (lib.mars_rope_frequencies(ctypes.byref(f), table) == 0) == ok
