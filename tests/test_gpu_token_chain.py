"""The token operators beside the verifier, as a training run uses them together: samples decoded under the mask of free
bases, verified, their violations counted, rewards turned into advantages, the policy loss and the gradient of the logits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2506_17506_amd as vl  # noqa: E402
from token_reference import U, Rows, advantages, near, policy  # noqa: E402
from vlgen import gen  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vl.load()


@pytest.mark.parametrize("first,pitch", [(0, 512), (1000, 1531)])
def test_from_logits_to_their_gradient(first, pitch):
    K = 12
    m = gen.Kernel(gen.LOOP3, 0xC4A1, 200, 150).mir
    O = m.n_occ
    hm = vl.vl_mir_create(m)
    hl = vl.vl_liveness(hm)
    ld = vl.pad_ld(O)
    cand = torch.zeros((K, ld), dtype=torch.int16, device="cuda")
    g = torch.Generator().manual_seed(7)
    logits = (torch.randn((K, O, pitch), generator=g) * 2).to(torch.bfloat16).cuda()
    masks = torch.zeros((K, O, 16), dtype=torch.int32, device="cuda")
    old = torch.zeros((K, O), device="cuda")
    step_mask = torch.zeros((K, 16), dtype=torch.int32, device="cuda")
    top, lp = torch.zeros((K, 4), dtype=torch.int32, device="cuda"), torch.zeros((K, 4), device="cuda")
    which = torch.arange(K, device="cuda")[:, None] % 3   # the best, the second, the third alternative
    for o in range(O):
        vl.vl_free_bases_multi([(hm, hl, cand[k], o) for k in range(K)], step_mask)
        vl.vl_token_logprobs(logits[:, o, first:first + 512], mask=step_mask, top_token=top, top_logprob=lp)
        # the alternative there is, or the best, or register 0 where nothing is free
        pick = torch.where(top.gather(1, which) >= 0, which, 0)
        cand[:, o] = top.gather(1, pick)[:, 0].clamp(min=0).to(torch.int16)
        old[:, o] = lp.gather(1, pick)[:, 0]
        masks[:, o] = step_mask
    # samples 0..5 as decoded: consistent and realizable wherever something was free throughout (a mask tests Safety at a value's
    # first occurrence only, so a value written again later may still clash there); the others with some registers changed
    free = (masks != 0).any(2).all(1).cpu().numpy()
    assert free.sum() >= 6
    for k in range(6, K):
        cand[k, torch.randint(0, O, (k,), generator=g).cuda()] ^= 3
    out = torch.zeros((K, 4), dtype=torch.int32, device="cuda")
    vl.vl_verify_batch(hm, hl, cand, K, ld, out)
    counts = torch.zeros((K, 8), dtype=torch.int32, device="cuda")
    vl.vl_count_violations_multi([(hm, hl, cand, K, ld, counts)])
    banks = torch.zeros(K, dtype=torch.int32, device="cuda")
    vl.vl_bank_conflicts(hm, cand, K, ld, 4, banks)
    status = out[:, 0].cpu().numpy()
    assert np.isin(status[:6][free[:6]], (0, 3)).all() and (status[:6] == 0).any() and (status[6:] != 0).any()
    extra = banks.float() * -0.001
    reward, adv = torch.zeros(K, device="cuda"), torch.zeros(K, device="cuda")
    w = (1.0, -0.02, -0.1, -0.05)
    vl.vl_group_advantages(counts, torch.tensor([0, K], dtype=torch.int32, device="cuda"), w, 1e-6, adv, reward=reward, extra=extra)
    r_want, a_want = advantages(counts.cpu().numpy(), extra.cpu().numpy(), [0, K], w, 1e-6)
    near(reward, r_want, U * np.abs(r_want) + 2.0 ** -40)
    near(adv, a_want, U * np.abs(a_want) + 2.0 ** -20)
    # the model as it is by now: other logits, scored at the samples' registers (their masks let the given one through)
    newer = (logits.float() + torch.randn(logits.shape, generator=g).cuda() * 0.2).to(torch.bfloat16)
    rows = newer.view(K * O, pitch)[:, first:first + 512]
    token = (cand[:, :O].int() & 0xFFFF).clamp(max=511).contiguous()
    stopped = torch.arange(O, device="cuda")[None] >= torch.tensor([O] * (K - 2) + [O // 3, 0], device="cuda")[:, None]
    token[stopped] = -1   # two samples that ended early
    token = token.view(-1)
    at = (token.clamp(min=0) >> 5).long()[:, None]
    mask = masks.view(K * O, 16).scatter(1, at, masks.view(K * O, 16).gather(1, at) | (1 << (token.clamp(min=0) & 31)).int()[:, None])
    n = K * O
    logprob, entropy, stat = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros((n, 2), device="cuda")
    vl.vl_token_logprobs(rows, token=token, mask=mask, logprob=logprob, entropy=entropy, stat=stat)
    want = Rows(rows, token, mask)
    near(logprob, want.logprob, want.logprob_err, "logprob")
    near(entropy, want.entropy, want.entropy_err, "entropy")
    start = torch.arange(0, n, O, device="cuda")
    length = torch.tensor([O] * (K - 2) + [O // 3, 0], dtype=torch.int32, device="cuda")
    weight = torch.full((K,), 1.0 / n, device="cuda")
    d_lp, stats = torch.zeros(n, device="cuda"), torch.zeros(24, dtype=torch.uint8, device="cuda")
    old = torch.where(torch.isfinite(old), old, -1.0).view(-1)
    ref = logprob + 0.01 * torch.randn(n, generator=g).cuda()
    vl.vl_policy_loss(logprob, old, start, length, adv, weight, d_lp, stats, -0.2, 0.2, logprob_ref=ref, kl=0.1, max_len=O)
    host = [x.cpu().numpy() for x in (logprob, old, ref, start, length, adv, weight)]
    p_grad, p_err, loss, loss_err, kls, kl_err, tokens, clipped = policy(*host, -0.2, 0.2, 0.1)
    outside = np.isnan(p_grad)
    near(d_lp, np.where(outside, 0, p_grad), np.where(outside, 0, p_err), "policy gradient")
    s = stats.cpu().numpy().view(vl.POLICY_STATS_DTYPE)[0]
    assert (s["n_token"], s["n_clipped"]) == (tokens, clipped) and clipped > 0 and tokens == (K - 2) * O + O // 3
    assert abs(s["loss"] - loss) <= loss_err and abs(s["kl"] - kls) <= kl_err
    bonus = torch.full((n,), -0.01 / n, device="cuda")
    grad = torch.full((n, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    vl.vl_token_logprobs_grad(rows, stat, grad, token=token, mask=mask, entropy=entropy, g_logprob=d_lp, g_entropy=bonus)
    d, err = want.grad(torch.bfloat16, d_lp, bonus)
    near(grad, d, err, "gradient of the logits")
    assert np.abs(d).max() > 0
    vl.vl_live_destroy(hl)
    vl.vl_mir_destroy(hm)
