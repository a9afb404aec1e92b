"""Advantages and the policy loss where numbers are infinite or missing, on the GPU: what is left of the others."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2506_17506_amd as vl  # noqa: E402
from test_gpu_policy_loss import call, check_out, device, make  # noqa: E402
from token_reference import U, advantages, near, policy  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vl.load()


@pytest.mark.parametrize("kl", [0.1, 0.0])
@pytest.mark.parametrize("m,n_tok", [(3, 7), (3, 600), (100, 700)])   # (one launch, and parts that are joined)
def test_a_token_that_the_model_cannot_emit_against_a_reference(m, n_tok, kl):
    """logprob -infinity, the reference finite: q = +infinity, exp(q) - q - 1 and exp(q) are infinite, and no other token's
    gradient is touched"""
    b = make([k * n_tok for k in range(m)], [n_tok] * m, m * n_tok, 11)
    b["adv"][:2], b["weight"][:2] = (1.5, -0.5), (0.25, 0.125)
    args = (b["start"], b["length"], b["adv"], b["weight"], -0.25, 0.25, kl)
    g, err = policy(b["lp"], b["old"], b["ref"], *args)[:2]
    at = [2, n_tok + 3]
    b["lp"][at] = -np.inf
    b["old"][at] = -1.0
    tokens, clipped = policy(b["lp"], b["old"], None, *args)[6:]
    d = device(b)
    grad, stats = torch.full_like(d["lp"], 77.0), torch.zeros(24, dtype=torch.uint8, device="cuda")
    call(d, grad, stats, kl=kl)
    s = stats.cpu().numpy().view(vl.POLICY_STATS_DTYPE)[0]
    assert (s["n_token"], s["n_clipped"]) == (tokens, clipped)
    assert s["kl"] == np.inf
    got = grad.cpu().numpy()
    if kl:
        assert s["loss"] == np.inf
        assert (got[at] == -np.inf).all()
    else:   # (the distance is only reported; exp(d) is 0 there, and the second's ratio is below the bound)
        some = [np.delete(b[k], at) for k in ("lp", "old")]
        short = b["length"].copy()
        short[:2] -= 1
        loss, loss_err = policy(*some, None, short.cumsum() - short, short, *args[2:])[2:4]
        clip = float(b["weight"][1]) * 0.5 * np.exp(-0.25)   # (what the second one adds: one rounding and the exponential's)
        assert abs(s["loss"] - (loss + clip)) <= loss_err + clip * 2.0 ** -20 + U * abs(loss + clip) and (got[at] == 0).all()
    others = np.ones(m * n_tok, bool)
    others[at] = False
    near(grad[torch.from_numpy(others).cuda()], g[others], err[others], "the others' gradient")


@pytest.mark.parametrize("n_tok", [7, 700])
def test_a_token_that_the_reference_cannot_emit(n_tok):
    """q = -infinity: exp(q) - q - 1 is infinite, exp(q) is 0"""
    m = 3
    b = make([k * n_tok for k in range(m)], [n_tok] * m, m * n_tok, 12)
    b["adv"][0], b["weight"][0] = 0.0, 0.25
    b["ref"][2] = -np.inf
    d = device(b)
    grad, stats = torch.full_like(d["lp"], 77.0), torch.zeros(24, dtype=torch.uint8, device="cuda")
    call(d, grad, stats, kl=0.5)
    s = stats.cpu().numpy().view(vl.POLICY_STATS_DTYPE)[0]
    assert s["loss"] == np.inf and s["kl"] == np.inf and grad[2].item() == 0.125 and grad.isfinite().all()


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("k", [2, 100, 300, 1025, 5000])   # (a wavefront, 256 and 1,024 threads per group; more than their registers hold)
@pytest.mark.parametrize("where", [0, 1, -1])
def test_a_reward_that_is_not_finite(k, where, bad):
    """mean and deviation of its group are not numbers, so neither is any of the group's advantages, wherever it stands; other
    groups keep theirs"""
    rng = np.random.default_rng(k)
    extra = rng.standard_normal(3 * k).astype(np.float32)
    extra[k:2 * k][where] = bad
    off = torch.tensor([0, k, 2 * k, 3 * k], dtype=torch.int32, device="cuda")
    reward, adv = torch.full((3 * k,), 77.0, device="cuda"), torch.full((3 * k,), 77.0, device="cuda")
    vl.vl_group_advantages(None, off, (1.0, 0.0, 0.0, 0.0), 1e-6, adv, reward=reward, extra=torch.from_numpy(extra).cuda())
    assert np.array_equal(reward.cpu().numpy(), extra, equal_nan=True)
    assert adv[k:2 * k].isnan().all()
    _, want = advantages(None, np.delete(extra, np.arange(k, 2 * k)), [0, k, 2 * k], (1.0, 0.0, 0.0, 0.0), 1e-6)
    near(torch.cat([adv[:k], adv[2 * k:]]), want, U * np.abs(want) + 2.0 ** -20, "the other groups")


@pytest.mark.parametrize("odd", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("m,n_tok,max_len", [(4, 9, None), (4, 9, 30000), (40, 1100, None)])   # (one workgroup, many slices, parts that are joined)
def test_weights_of_samples_without_tokens(m, n_tok, max_len, odd):
    """weight = 1 / (samples * len) is infinite for a sample that was stopped before its first token, or lies past the arrays: it adds
    nothing"""
    length = np.full(m, n_tok)
    length[[0, m - 1]] = 0
    start = length.cumsum() - length
    start[1], b_n = 2 ** 40, int(length.sum())   # (the second sample's tokens are not there)
    b = make(start, length, b_n, 13)
    b["adv"][[0, 1, m - 1]] = (1.0, -1.0, 0.0)
    b["weight"][[0, 1, m - 1]] = odd
    d = device(b)
    grad, stats = torch.full_like(d["lp"], 77.0), torch.full((24,), 255, dtype=torch.uint8, device="cuda")
    call(d, grad, stats, max_len=max_len)
    check_out(b, grad, stats)
