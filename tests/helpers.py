"""Shared test helpers: small model shapes and an oracle-side runner (CPU only); the rotation's
frequencies with 60 digits."""
from decimal import Decimal, localcontext

import torch

import oracle
from paper_2511_11373_b200 import workloads as wl

SMALL = dict(n_layers=2, hidden=64, n_q_heads=4, n_kv_heads=2, head_dim=16, n_experts=4, top_k=2,
             expert_inter=32, vocab=50, qk_norm=1, rope_theta=1e4, rms_eps=1e-6)


def ocfg(model: dict) -> oracle.Config:
    return oracle.Config(**model)


def bf16_bits(t: torch.Tensor) -> torch.Tensor:
    return t.contiguous().view(torch.int16)


def fresh_cache(model, n_pages, page_size, seed=0, fill=True):
    return wl.make_kv_pools(model, n_pages, page_size, seed=seed, device="cpu", fill=fill)


def rel_l2(a: torch.Tensor, b: torch.Tensor) -> float:
    a, b = a.double(), b.double()
    return float((a - b).norm() / b.norm().clamp_min(1e-30))


TWO_PI = Decimal("6.28318530717958647692528676655900576839433879875021164194988918")


def exact_frequencies(rotary, scaling, theta, factor=8.0, trained=32768.0, fast=32.0, slow=1.0):
    """The frequencies with 60 digits."""
    with localcontext() as ctx:
        ctx.prec = 60
        d, theta, factor, trained, fast, slow = (Decimal(v) for v in (rotary, theta, factor, trained, fast, slow))
        if scaling == 2:
            theta *= factor ** (d / (d - 2))
        out = []
        for i in range(rotary // 2):
            v = theta ** (-2 * i / d)
            if scaling == 1:
                v /= factor
            if scaling == 3:
                keep = min(Decimal(1), max(Decimal(0), (trained * v / TWO_PI - slow) / (fast - slow)))
                v *= keep + (1 - keep) / factor
            out.append(v)
        return out
