"""Advantages and the policy loss on the GPU against their definitions in 64 bits (token_reference.py)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2506_17506_amd as vl  # noqa: E402
from token_reference import U, advantages, near, policy  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vl.load()


W = (1.0, -0.02, -0.1, -0.003)


def some_counts(n, seed):
    rng = np.random.default_rng(seed)
    c = np.zeros((n, 8), np.int32)
    for word, most in ((1, 40), (2, 5), (3, 100000)):
        c[:, word] = np.where(rng.random(n) < 0.4, rng.integers(1, most, n), 0)
    c[:, 0] = (c[:, 1] > 0) | (c[:, 2] > 0) << 1 | (c[:, 3] > 0) << 2
    c[:, 5:] = -1
    return c


def check_advantages(counts, extra, off, weights=W, eps=1e-6, stream=None):
    n = len(counts if counts is not None else extra)
    reward, adv = torch.full((n,), 77.0, device="cuda"), torch.full((n,), 77.0, device="cuda")
    vl.vl_group_advantages(None if counts is None else torch.from_numpy(counts).cuda(), torch.from_numpy(np.asarray(off, np.uint32).view(np.int32)).cuda(),
                           weights, eps, adv, reward=reward, extra=None if extra is None else torch.from_numpy(extra).cuda(), stream=stream)
    r, a = advantages(counts, extra, np.asarray(off, np.int64), weights, eps)
    out = np.isnan(a)
    assert (reward.cpu().numpy()[out] == 77).all() and (adv.cpu().numpy()[out] == 77).all()
    r, a = np.where(out, 77, r), np.where(out, 77, a)
    # rewards: products and sums in 64 bits and one rounding; advantages: the distance to the mean is off by 2^-50 of the largest reward
    # over a deviation that is at least 1e-9 of it wherever it is not 0, and one rounding
    near(reward, r, U * np.abs(r) + 2.0 ** -40, "reward")
    near(adv, a, U * np.abs(a) + 2.0 ** -20, "advantage")
    return adv


@pytest.mark.parametrize("k", [1, 2, 3, 63, 64, 65, 100, 255, 256, 257, 1000, 1024, 1025, 4097, 65535])
def test_group_sizes(k):
    c = some_counts(2 * k, k)
    check_advantages(c, None, [0, k, 2 * k])


@pytest.mark.parametrize("groups", [1, 2, 300, 70000])
def test_many_ragged_groups(groups):
    rng = np.random.default_rng(groups)
    size = rng.integers(0, 9, groups)   # some are empty
    off = 5 + np.concatenate([[0], size.cumsum()])   # the first five samples and the last three belong to none
    n = int(off[-1]) + 3
    check_advantages(some_counts(n, groups), rng.standard_normal(n).astype(np.float32), off)


def test_rewards_of_one_kind():
    n = 500
    rng = np.random.default_rng(1)
    check_advantages(None, rng.standard_normal(n).astype(np.float32), [0, 200, 500])
    check_advantages(some_counts(n, 2), None, [0, 500], weights=(0, 0, 0, 0))
    equal = some_counts(n, 3)
    equal[:] = equal[7]
    adv = check_advantages(equal, None, [0, 3, 499, 500], weights=(0.1, -0.3, 0.7, -0.1))
    assert (adv == 0).all()   # exactly
    adv = check_advantages(None, np.full(n, 0.1, np.float32), [0, 500])
    assert (adv == 0).all()


def test_only_one_output_and_offsets_past_the_samples():
    n = 64
    c = some_counts(n, 5)
    adv = torch.full((n,), 77.0, device="cuda")
    off = torch.tensor([0, 60, 100, 2 ** 31 - 1], dtype=torch.int32, device="cuda")   # samples at n and above are not there
    vl.vl_group_advantages(torch.from_numpy(c).cuda(), off, W, 1e-6, adv)
    _, a = advantages(c, None, [0, 60, 100, 2 ** 31 - 1], W, 1e-6)
    near(adv, a, U * np.abs(a) + 2.0 ** -20)


def make(start, length, n, seed, ref=True):
    rng = np.random.default_rng(seed)
    m = len(start)
    lp = np.log(rng.random(n) ** 2 + 1e-6).astype(np.float32)
    old = (lp + 0.3 * rng.standard_normal(n)).astype(np.float32)
    far = (lp + np.where(rng.random(n) < 0.5, 0.01, 1.0) * rng.standard_normal(n)).astype(np.float32) if ref else None
    adv = rng.standard_normal(m).astype(np.float32)
    adv[rng.random(m) < 0.1] = 0
    weight = (rng.random(m) / max(1, np.sum(length))).astype(np.float32)
    return dict(lp=lp, old=old, ref=far, start=np.asarray(start, np.int64), length=np.asarray(length, np.int32), adv=adv, weight=weight)


def device(b):
    return {k: None if v is None else torch.from_numpy(v).cuda() for k, v in b.items()}


def call(d, grad, stats, lo=-0.25, hi=0.25, kl=0.1, **more):
    vl.vl_policy_loss(d["lp"], d["old"], d["start"], d["length"], d["adv"], d["weight"], grad, stats, lo, hi, logprob_ref=d["ref"], kl=kl, **more)


def check_policy(b, lo=-0.25, hi=0.25, kl=0.1, in_place=False, **more):
    d = device(b)
    kl = kl if b["ref"] is not None else 0.0
    grad = d["lp"] if in_place else torch.full_like(d["lp"], 77.0)
    stats = torch.full((24,), 255, dtype=torch.uint8, device="cuda")
    call(d, grad, stats, lo, hi, kl, **more)
    check_out(b, grad, stats, lo, hi, kl, rest=b["lp"] if in_place else None)


def check_out(b, grad, stats, lo=-0.25, hi=0.25, kl=0.1, rest=None):
    g, err, loss, loss_err, kls, kl_err, tokens, clipped = policy(b["lp"], b["old"], b["ref"], b["start"], b["length"], b["adv"], b["weight"], lo, hi, kl)
    outside = np.isnan(g)
    got = grad.cpu().numpy()
    assert (got[outside] == (77.0 if rest is None else rest[outside])).all()
    near(grad[torch.from_numpy(~outside).cuda()], g[~outside], err[~outside], "grad")
    s = stats.cpu().numpy().view(vl.POLICY_STATS_DTYPE)[0]
    assert (s["n_token"], s["n_clipped"]) == (tokens, clipped)
    assert abs(s["loss"] - loss) <= loss_err, (s["loss"], loss, loss_err)
    assert abs(s["kl"] - kls) <= kl_err, (s["kl"], kls, kl_err)


@pytest.mark.parametrize("ref", [False, True])
@pytest.mark.parametrize("n_tok", [1, 2, 3, 4, 5, 63, 64, 255, 1023, 1024, 1025, 5261, 20011])
def test_lengths(n_tok, ref):
    m = 5
    gap = n_tok % 3   # starts of every alignment
    check_policy(make([gap + k * (n_tok + gap) for k in range(m)], [n_tok] * m, m * (n_tok + gap) + 7, n_tok, ref))


@pytest.mark.parametrize("m", [1, 2, 100, 1500, 70000])
def test_many_ragged_samples(m):
    rng = np.random.default_rng(m)
    length = np.minimum(rng.integers(0, 60, m), rng.integers(0, 60, m))
    if m < 2000:
        length[rng.integers(0, m)] = 30011   # one far longer than the others
    start = np.concatenate([[0], length.cumsum()[:-1]])
    order = rng.permutation(m)   # samples in any order
    check_policy(make(start[order], length[order], int(length.sum()) + 1, m))


@pytest.mark.parametrize("m,n_tok", [(1, 1), (1, 16384), (16, 1000), (17, 900), (32, 512), (33, 400), (1, 16385), (8, 2048), (4, 4096)])
def test_small_batches(m, n_tok):
    """around what one workgroup takes alone"""
    for ref in (False, True):
        b = make([k * n_tok for k in range(m)], [n_tok - (k % 3 if n_tok > 3 else 0) for k in range(m)], m * n_tok, m, ref)
        check_policy(b)
        check_policy(b, max_len=n_tok)


def test_no_tokens_at_all():
    check_policy(make([0, 3], [0, 0], 5, 1))


@pytest.mark.parametrize("max_len", [1, 1000, 2 ** 32 - 1])
def test_the_longest_length_is_a_hint(max_len):
    check_policy(make([0, 9000], [9000, 17], 9017, 3), max_len=max_len)


def test_in_place():
    check_policy(make([2, 500], [400, 700], 1300, 3), in_place=True)


def test_lengths_past_the_arrays():
    """tokens at n and above are not there; a start past it has none"""
    check_policy(make([90, 10, 2 ** 40, 2 ** 62], [1000, 20, 5, 2 ** 31 - 1], 100, 3))


def test_bounds():
    """no clipping, all of one side clipped, numbers exactly at a bound and one step beside it"""
    b = make([0, 300], [300, 300], 600, 4)
    check_policy(b, lo=-np.inf, hi=np.inf)
    check_policy(b, lo=0.0, hi=0.0)
    b["old"] = np.zeros(600, np.float32)
    at = np.float32([-0.25, np.nextafter(np.float32(-0.25), np.float32(-1)), np.nextafter(np.float32(-0.25), np.float32(0)),
                     0.25, np.nextafter(np.float32(0.25), np.float32(1)), np.nextafter(np.float32(0.25), np.float32(0))])
    b["lp"] = np.tile(at, 100)
    b["adv"][:] = [1.0, -1.0]
    check_policy(b)
    # a difference that 32 bits would round onto the bound
    b["lp"][:] = np.float32(0.25)
    b["old"][:] = np.float32(-1e-9)
    check_policy(b)


def test_extreme_log_probabilities():
    b = make([0, 8], [8, 8], 16, 5, ref=False)
    b["adv"][:] = [1.5, -1.5]
    b["lp"] = np.tile(np.float32([-np.inf, -200, -1e-30, 0, -5, -1e30, -80, -3]), 2)
    b["old"] = np.tile(np.float32([-1, -1, -70, -1e-38, -1e5, -2, -1, -np.inf]), 2)
    d = device(b)
    grad, stats = torch.zeros(16, device="cuda"), torch.zeros(24, dtype=torch.uint8, device="cuda")
    call(d, grad, stats, kl=0.0)
    g, err, *_ = policy(b["lp"], b["old"], None, b["start"], b["length"], b["adv"], b["weight"], -0.25, 0.25, 0.0)
    with np.errstate(over="ignore"):
        g = g.astype(np.float32).astype(float)   # (what 32 bits do not hold)
    near(grad, g, np.where(np.isfinite(err), err, 0))


@pytest.mark.parametrize("n_tok", [7, 700])   # (one launch, and parts that are joined)
def test_factors_of_zero(n_tok):
    # ratios and distances that 32 bits do not hold, in terms whose factor is 0: they add nothing
    m = 100 if n_tok > 100 else 3
    b = make([k * n_tok for k in range(m)], [n_tok] * m, m * n_tok, 8)
    b["adv"][:3], b["weight"][:3] = (0.0, -2.0, 0.5), (0.25, 0.0, 0.125)
    b["old"][:2 * n_tok] = b["lp"][:2 * n_tok] - 100
    near_ref, b["ref"] = b["ref"], None
    check_policy(b)
    b["ref"] = near_ref
    check_policy(b)
    b["ref"][n_tok:2 * n_tok] += 120   # in the sample without weight
    check_policy(b)
    b["ref"][0] += 120
    d = device(b)
    grad, stats = torch.full_like(d["lp"], 77.0), torch.empty(24, dtype=torch.uint8, device="cuda")
    call(d, grad, stats, kl=0.0)   # the distance is only reported
    g, err, loss, loss_err = policy(b["lp"], b["old"], b["ref"], b["start"], b["length"], b["adv"], b["weight"], -0.25, 0.25, 0.0)[:4]
    near(grad, g, err, "grad")
    s = stats.cpu().numpy().view(vl.POLICY_STATS_DTYPE)[0]
    assert abs(s["loss"] - loss) <= loss_err and s["kl"] == np.inf


def test_gradient_against_differences():
    """of the loss in 64 bits, which check_policy holds the kernel's to: h = 2^-12 leaves h^2 / 6 times the third derivative"""
    b = make([0], [40], 40, 6)
    d = device(b)
    grad, stats = torch.zeros(40, device="cuda"), torch.zeros(24, dtype=torch.uint8, device="cuda")
    call(d, grad, stats)
    h = 2.0 ** -12
    for i in range(40):
        if abs(abs(b["lp"][i] - b["old"][i]) - 0.25) < 0.001:
            continue   # (the loss has a corner there)
        both = []
        for s in (h, -h):
            lp = b["lp"].astype(np.float64)
            lp[i] += s
            both.append(policy(lp, b["old"], b["ref"], b["start"], b["length"], b["adv"], b["weight"], -0.25, 0.25, 0.1)[2])
        scale = abs(b["weight"][0]) * (abs(b["adv"][0]) + 0.1) * 30
        assert abs((both[0] - both[1]) / (2 * h) - grad[i].item()) < scale * (h * h + 2.0 ** -20)


def test_streams_and_a_recorded_pass():
    batches = [make([0, 40000, 40100], [40000, 100, 30000], 70100, k) for k in (1, 2)]
    ds = [device(b) for b in batches]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for turn in range(4):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                grad, stats = torch.full_like(ds[k]["lp"], 77.0), torch.zeros(24, dtype=torch.uint8, device="cuda")
            call(ds[k], grad, stats, stream=streams[k])
            outs.append((k, grad, stats))
    torch.cuda.synchronize()
    for k, grad, stats in outs:
        check_out(batches[k], grad, stats)
    d = {k: v.clone() for k, v in ds[0].items()}
    grad, stats = torch.zeros_like(d["lp"]), torch.zeros(24, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(d, grad, stats)
    for k in (1, 0, 1):
        for name in d:
            d[name].copy_(ds[k][name])
        grad.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        check_out(batches[k], grad, stats)


def test_equal_calls_give_equal_bits():
    d = device(make([0, 40000], [40000, 30000], 70000, 1))
    got = []
    for _ in range(3):
        grad, stats = torch.zeros_like(d["lp"]), torch.zeros(24, dtype=torch.uint8, device="cuda")
        call(d, grad, stats)
        got.append((grad.cpu(), stats.cpu()))
    assert all((g == got[0][0]).all() and (s == got[0][1]).all() for g, s in got)


def test_refusals_of_the_binding():
    d = device(make([0], [40], 40, 6))
    grad, stats = torch.zeros(40, device="cuda"), torch.zeros(24, dtype=torch.uint8, device="cuda")

    def code(g=grad, st=stats, lo=-0.25, kl=0.1, **change):
        with pytest.raises(vl.VlError) as err:
            call({**d, **change}, g, st, lo=lo, kl=kl)
        return err.value.code
    assert code(g=grad[:39]) == -2 and code(g=grad.half()) == -3 and code(g=None) == -1 and code(g=grad.cpu()) == -7
    assert code(st=stats[:20]) == -2 and code(old=d["old"].cpu()) == -7 and code(old=d["old"][::2]) == -2 and code(lp=None) == -1
    assert code(start=d["start"].int()) == -3 and code(length=d["length"].long()) == -3 and code(adv=None) == -1
    assert code(weight=d["weight"].double()) == -3 and code(lo=0.5) == -3 and code(ref=None) == -1 and code(kl=float("nan")) == -3
    assert code(start=d["start"][:0], length=d["length"][:0], adv=d["adv"][:0], weight=d["weight"][:0]) == -2
    c, adv = torch.from_numpy(some_counts(8, 1)).cuda(), torch.zeros(8, device="cuda")
    off = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    for args, want in (((c[:7], off, W, 1e-6, adv), -2), ((c.long(), off, W, 1e-6, adv), -3), ((c, off.cpu(), W, 1e-6, adv), -7), ((c, off[:1], W, 1e-6, adv), -2),
                       ((c, off, W, 0.0, adv), -3), ((c, off, (1e300, 0, 0, 0), 1e-6, adv), -3), ((None, off, W, 1e-6, adv), -1), ((c, off, W, 1e-6, None), -1), ((c[:0], off, W, 1e-6, adv[:0]), -2)):
        with pytest.raises(vl.VlError) as err:
            vl.vl_group_advantages(*args)
        assert err.value.code == want, args
    torch.cuda.synchronize()
    assert (grad == 0).all() and (adv == 0).all()
