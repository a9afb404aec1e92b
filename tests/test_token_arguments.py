"""What the token operators refuse, at the C entry points: before anything is read or launched, so without a GPU.  And the
reference of their GPU tests against torch's own functions."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2506_17506_amd as vl
from paper_2506_17506_amd import binding
from token_reference import Rows, words_of

NULL, SHAPE, RANGE = -1, -2, -3
MEM = C.create_string_buffer(4096)
P = (C.addressof(MEM) + 63) & ~63   # never read


def rows(**change):
    a = binding._TokenRows(P, 64, P, 2, P, 4, 64, vl.VL_BF16, 1.0)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def scores(**change):
    o = binding._TokenScores(P, P, P, P, P, 4, 0)
    for k, v in change.items():
        setattr(o, k, v)
    return o


BAD_ROWS = [
    (dict(logits=None), NULL), (dict(ld=63), SHAPE), (dict(mask_ld=1), SHAPE), (dict(n_row=0), SHAPE), (dict(n_row=1 << 31), SHAPE),
    (dict(n_vocab=0), RANGE), (dict(n_vocab=(1 << 24) + 1, ld=1 << 25, mask=None), RANGE), (dict(type=3), RANGE),
    (dict(scale=0.0), RANGE), (dict(scale=-1.0), RANGE), (dict(scale=float("nan")), RANGE), (dict(scale=float("inf")), RANGE),
    (dict(logits=P + 1), SHAPE), (dict(logits=P + 2, type=vl.VL_F32), SHAPE), (dict(mask=P + 2), SHAPE), (dict(token=P + 1), SHAPE),
]


@pytest.mark.parametrize("change,code", BAD_ROWS)
def test_rows_refused(change, code):
    lib, need = vl.load(), C.c_uint64(77)
    a, o = rows(**change), scores()
    assert lib.vl_token_logprobs(C.byref(a), C.byref(o), None, 0, None) == code
    assert lib.vl_token_logprobs_work(C.byref(a), C.byref(o), C.byref(need)) == code and need.value == 77
    assert lib.vl_token_logprobs_grad(C.byref(a), P, P, P, P, P, 1 << 25, None) == code


@pytest.mark.parametrize("change,code", [
    (dict(logprob=None, entropy=None, stat=None, top_token=None, top_logprob=None, n_top=0), NULL), (dict(n_top=0), NULL),
    (dict(top_token=None, top_logprob=None), NULL), (dict(n_top=33), RANGE), (dict(reserved0=1), RANGE), (dict(logprob=P + 2), SHAPE),
    (dict(entropy=P + 1), SHAPE), (dict(stat=P + 3), SHAPE), (dict(top_token=P + 2), SHAPE), (dict(top_logprob=P + 2), SHAPE)])
def test_scores_refused(change, code):
    lib, a, o = vl.load(), rows(), scores(**change)
    assert lib.vl_token_logprobs(C.byref(a), C.byref(o), None, 0, None) == code


def test_missing_parts():
    lib, a, o = vl.load(), rows(token=None), scores()
    assert lib.vl_token_logprobs(C.byref(a), C.byref(o), None, 0, None) == NULL   # a log probability of no token
    assert lib.vl_token_logprobs(None, C.byref(o), None, 0, None) == NULL
    assert lib.vl_token_logprobs(C.byref(a), None, None, 0, None) == NULL
    assert lib.vl_token_logprobs_work(C.byref(a), C.byref(o), None) == NULL
    grad = lib.vl_token_logprobs_grad
    assert grad(None, P, P, P, P, P, 64, None) == NULL
    assert grad(C.byref(a), P, P, P, None, P, 64, None) == NULL                    # no token
    a = rows()
    for k in range(5):
        args = [P] * 5
        args[k] = None
        if k in (0, 1, 4):   # stat, entropy (with g_entropy), grad
            assert grad(C.byref(a), *args, 64, None) == NULL, k
    assert grad(C.byref(a), P, P, None, None, P, 64, None) == NULL
    assert grad(C.byref(a), P, P, P, P, P, 63, None) == SHAPE
    assert grad(C.byref(a), P, P, P, P, P + 1, 64, None) == SHAPE
    assert grad(C.byref(a), P + 2, P, P, P, P, 64, None) == SHAPE


def test_work_too_small_or_not_aligned():
    lib, need = vl.load(), C.c_uint64()
    a, o = rows(n_row=1, n_vocab=1 << 20, ld=1 << 20, mask=None), scores()
    assert lib.vl_token_logprobs_work(C.byref(a), C.byref(o), C.byref(need)) == 0
    if need.value:
        assert lib.vl_token_logprobs(C.byref(a), C.byref(o), None, 0, None) == NULL
        assert lib.vl_token_logprobs(C.byref(a), C.byref(o), P, need.value - 1, None) == SHAPE
        assert lib.vl_token_logprobs(C.byref(a), C.byref(o), P + 8, need.value, None) == SHAPE


def test_advantages_refused():
    f = vl.load().vl_group_advantages

    def code(counts=P, extra=P, n=8, off=P, n_group=2, weights=(1, 2, 3, 4), eps=1e-6, reward=P, advantage=P):
        w = None if weights is None else C.byref(binding._RewardWeights(*weights))
        return f(counts, extra, n, off, n_group, w, eps, reward, advantage, None)
    assert code(counts=None, extra=None) == NULL
    assert code(off=None) == NULL and code(weights=None) == NULL and code(reward=None, advantage=None) == NULL
    assert code(n=0) == SHAPE and code(n=1 << 31) == SHAPE and code(n_group=0) == SHAPE and code(n_group=1 << 31) == SHAPE
    assert code(extra=P + 1) == SHAPE and code(counts=P + 2) == SHAPE
    for w in (float("nan"), float("inf")):
        for k in range(4):
            assert code(weights=[w if j == k else 1.0 for j in range(4)]) == RANGE
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert code(eps=eps) == RANGE


def test_policy_refused():
    lib = vl.load()

    def code(grad=P, stats=P, work=P, work_bytes=1 << 40, **change):
        b = binding._PolicyBatch(P, P, P, 100, P, P, P, P, 4, 10, -0.2, 0.2, 0.1, 0)
        for k, v in change.items():
            setattr(b, k, v)
        return lib.vl_policy_loss(C.byref(b), grad, stats, work, work_bytes, None)
    for name in ("logprob", "logprob_old", "logprob_ref", "start", "len", "advantage", "weight"):
        assert code(**{name: None}) == NULL, name
        assert code(**{name: P + 2}) == SHAPE, name
    assert code(start=P + 4) == SHAPE
    many = dict(n=1 << 30, n_sample=1000)   # (few tokens need no work)
    assert code(grad=None) == NULL and code(stats=None) == NULL and code(work=None, **many) == NULL
    assert code(grad=P + 2) == SHAPE and code(stats=P + 4) == SHAPE and code(work=P + 8, **many) == SHAPE and code(work_bytes=0, **many) == SHAPE
    assert code(n=0) == SHAPE and code(n=1 << 60) == SHAPE and code(n_sample=0) == SHAPE and code(n_sample=1 << 31) == SHAPE
    for change in (dict(log_lo=0.3), dict(log_lo=float("nan")), dict(log_hi=float("nan")), dict(kl=float("nan")), dict(kl=float("inf")), dict(reserved0=1)):
        assert code(**change) == RANGE, change
    assert lib.vl_policy_loss(None, P, P, P, 1 << 40, None) == NULL
    assert lib.vl_policy_loss_work(None, C.byref(C.c_uint64())) == NULL


def test_the_binding_refuses_host_tensors():
    with pytest.raises(vl.VlError) as e:
        vl.vl_token_logprobs(torch.zeros(2, 4), entropy=torch.zeros(2))
    assert e.value.code == -7


def test_reference_against_torch():
    """the definitions as written out for the GPU tests, against log_softmax and its gradient in 64 bits"""
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((6, 40), generator=gen, dtype=torch.float64).float()
    bits = np.random.default_rng(1).random((6, 40)) < 0.5
    bits[:, 3] = True
    t = torch.full((6,), 3, dtype=torch.int32)
    want = Rows(x, t, words_of(bits), 0.7, top=4)
    leaf = x.double().requires_grad_()
    lp = torch.log_softmax((leaf * float(np.float32(0.7))).masked_fill(~torch.from_numpy(bits), float("-inf")), 1)
    p = lp.exp()
    h = -(p * lp.masked_fill(p == 0, 0.0)).sum(1)
    assert np.abs(lp[:, 3].detach().numpy() - want.logprob).max() < 1e-12 and np.abs(h.detach().numpy() - want.entropy).max() < 1e-12
    g, e = torch.randn(6, generator=gen), torch.randn(6, generator=gen)
    (lp[:, 3] * g.double() + h * e.double()).sum().backward()
    d, _ = want.grad(torch.float32, g, e)
    assert np.abs(leaf.grad.numpy() - d).max() < 1e-12
    top = lp.topk(4, 1)
    assert (top.indices.numpy() == want.top_token).all() and np.abs(top.values.detach().numpy() - want.top_logprob).max() < 1e-12
