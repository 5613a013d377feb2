"""Policy-update operators, host side (no device): sizes, refusals that are decided before any CUDA call, and the
binding's checks of tensors."""
import ctypes

import pytest
import torch

from paper_2511_11373_b200 import binding


@pytest.fixture(scope="module")
def lib():
    from paper_2511_11373_b200 import build
    build.build()
    return binding.lib()


@pytest.mark.parametrize("hidden,vocab,n", [(256, 1024, 4), (2048, 151936, 4096), (8, 1, 1), (264, 1013, 37), (0, 0, 0)])
def test_workspace_sizes(lib, hidden, vocab, n):
    b = lib.mars_update_workspace_bytes(hidden, vocab, n)
    assert b > 0 and b % 256 == 0
    if n:
        assert lib.mars_update_workspace_bytes(hidden, vocab, n + 256) > b * 0.99
        # the logits are never held: one vocabulary piece of the gradient, and fp32 sums of d_hidden, whatever the vocabulary
        rows = -(-n // 256) * 256
        assert b <= (512 << 20) + rows * (2048 * 2 + 8 * -(-vocab // 256) + 17 * 4 * hidden + 2 * hidden + 64) + 65536


@pytest.mark.parametrize("hidden,vocab,n", [(0, 10, 1), (12, 10, 1), (8, 0, 1), (8, 10, 0), (-8, 10, 1), (8, -1, 1), (8, 10, -1),
                                            (4, 10, 1), (0, 0, 5)])
def test_unsupported_shapes_have_no_workspace_and_no_handle(lib, hidden, vocab, n):
    assert lib.mars_update_workspace_bytes(hidden, vocab, n) == 0
    out = ctypes.c_void_p()
    assert lib.mars_update_create(hidden, vocab, n, ctypes.c_void_p(256), 1 << 40, ctypes.byref(out)) == 2
    assert not out.value


def test_null_handles_and_bad_workspaces_are_refused(lib):
    out = ctypes.c_void_p()
    assert lib.mars_update_create(8, 10, 1, None, 1 << 30, ctypes.byref(out)) == 1
    assert lib.mars_update_create(8, 10, 1, ctypes.c_void_p(128), 1 << 30, ctypes.byref(out)) == 1      # alignment
    assert lib.mars_update_create(8, 10, 1, ctypes.c_void_p(256), 256, ctypes.byref(out)) == 1          # too small
    assert lib.mars_update_create(8, 10, 1, ctypes.c_void_p(256), 1 << 30, None) == 1
    assert lib.mars_update_free(None) == 6 and lib.mars_update_poll_status(None) == 6
    assert lib.mars_logprob(None, None, 1, None, 8, None, None, 1.0, None, None) == 6
    assert lib.mars_logprob_grad(None, None, 1, None, 8, None, None, 1.0, None, None, None, 8, None, 1, 0) == 6
    assert lib.mars_expert_matmul(None, None, 1, 1, 8, 8, None, 8, None, None, None, 8, 1) == 6
    assert lib.mars_expert_matmul_dx(None, None, 1, 1, 8, 8, None, 8, None, None, None, 8, 1) == 6
    assert lib.mars_expert_matmul_dw(None, None, 1, 1, 8, 8, None, 8, None, 8, None, None, 1, 0) == 6
    assert lib.mars_grads_free(None) == 6 and lib.mars_grads_norm(None, None, None) == 6
    assert lib.mars_grads_clip(None, None, 1.0, None) == 6


def entry(grad, out, numel, type_=0):
    return binding.mars_grad_t(grad, out, numel, type_, 0)


@pytest.mark.parametrize("entries", [
    [entry(0, 4096, 1)], [entry(4096, 0, 1)], [entry(4096, 4096, -1)], [entry(4096, 4096, 4, 3)], [entry(4096, 4096, 4, -1)],
    [entry(4098, 4098, 4, 0)],                                            # fp32 off its alignment
    [entry(4097, 4097, 4, 1)],
    [entry(4096, 4100, 4)],                                               # out overlaps its own gradient in part
    [entry(4096, 4096, 4), entry(4096, 4096, 4)],                         # the same tensor twice, in place
    [entry(4096, 8192, 4), entry(4096, 8192, 4)],                         # the same out twice
    [entry(4096, 4096, 4), entry(4108, 4108, 4)],                         # neighbours that share a value
    [entry(4096, 8192, 4), entry(8200, 12288, 4)],                        # one's out is another's gradient
    [entry(4096, 4096, 64), entry(4100, 9000, 1)],                        # a gradient inside another's out
])
def test_gradient_lists_that_cannot_be_scaled_are_refused(lib, entries):
    n = lib.mars_grads_bytes(len(entries))
    assert n > 0 and n % 256 == 0
    table = (binding.mars_grad_t * len(entries))(*entries)
    out = ctypes.c_void_p()
    assert lib.mars_grads_create(table, len(entries), ctypes.c_void_p(256), n, ctypes.byref(out)) == 1
    assert not out.value


def test_gradient_list_sizes(lib):
    assert lib.mars_grads_bytes(0) == 0 and lib.mars_grads_bytes(-1) == 0 and lib.mars_grads_bytes((1 << 20) + 1) == 0
    assert lib.mars_grads_bytes(435) < 64 << 10
    out = ctypes.c_void_p()
    one = (binding.mars_grad_t * 1)(entry(4096, 4096, 4))
    assert lib.mars_grads_create(one, 1, ctypes.c_void_p(256), 64, ctypes.byref(out)) == 1
    assert lib.mars_grads_create(one, 1, ctypes.c_void_p(64), 1 << 20, ctypes.byref(out)) == 1
    assert lib.mars_grads_create(None, 1, ctypes.c_void_p(256), 1 << 20, ctypes.byref(out)) == 1


def test_the_binding_refuses_tensors_of_another_kind():
    class Fake:                                       # stands for a handle: the checks come before the library
        hidden, vocab, max_tokens, handle = 8, 10, 4, None
        device = torch.device("cpu")

    f = Fake()
    ok = dict(hidden=torch.zeros(4, 8, dtype=torch.bfloat16), lm_head=torch.zeros(10, 8, dtype=torch.bfloat16),
              targets=torch.zeros(4, dtype=torch.int32), lp=torch.zeros(4), lse=torch.zeros(4))

    def call(**kw):
        a = dict(ok, **kw)
        return binding.mars_logprob(f, a["hidden"], a["lm_head"], a["targets"], 1.0, a["lp"], a["lse"])

    for bad in (dict(hidden=torch.zeros(4, 8)), dict(hidden=torch.zeros(4, 16, dtype=torch.bfloat16)),
                dict(hidden=torch.zeros(8, 4, dtype=torch.bfloat16).t()), dict(lm_head=torch.zeros(9, 8, dtype=torch.bfloat16)),
                dict(lm_head=torch.zeros(10, 16, dtype=torch.bfloat16)[:, :8]), dict(targets=torch.zeros(4, dtype=torch.int64)),
                dict(targets=torch.zeros(5, dtype=torch.int32)), dict(lp=torch.zeros(4, dtype=torch.float64)), dict(lse=torch.zeros(3)),
                dict(hidden=torch.zeros(1, 8, dtype=torch.bfloat16).expand(4, 8))):
        with pytest.raises(ValueError):
            call(**bad)
    w, off = torch.zeros(3, 16, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    x, y = torch.zeros(5, 8, dtype=torch.bfloat16), torch.zeros(5, 16)
    for args in ((x, off[:3], w, y), (x, off.long(), w, y), (x.float(), off, w, y), (x, off, w[0], y), (x, off, w, y[:, :8]),
                 (x, off, w, y.half()), (x[:4], off, w, y)):
        with pytest.raises(ValueError):
            binding.mars_expert_matmul(f, *args)
    with pytest.raises(ValueError):
        binding.mars_expert_matmul_dx(f, x, off, w, x)
    with pytest.raises(ValueError):
        binding.mars_expert_matmul_dw(f, y.bfloat16(), x, off, w.half())
    for grads, outs in (([], None), ([torch.zeros(3)], [torch.zeros(4)]), ([torch.zeros(3)], [torch.zeros(3).half()]),
                        ([torch.zeros(3, dtype=torch.float64)], None), ([torch.zeros(4, 4)[:, :2]], None), ([torch.zeros(3)], None)):
        with pytest.raises(ValueError):
            binding.GradList(grads, outs)


def test_the_gradient_with_log_probs_refuses_a_null_handle(lib):
    assert lib.mars_logprob_grad_lp(None, None, 1, None, 8, None, None, 1.0, None, None, None, None, 8, None, 1, 0) == 6
