"""Token scores and their gradient on the GPU against the definitions in 64 bits (token_reference.py)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2506_17506_amd as vl  # noqa: E402
from token_reference import Rows, near, words_of  # noqa: E402

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vl.load()


def scores(x, token=None, mask=None, scale=1.0, top=0, stream=None):
    """every output, preset to something else"""
    n = x.shape[0]
    out = dict(entropy=torch.full((n,), 7.0, device="cuda"), stat=torch.full((n, 2), 7.0, device="cuda"))
    if token is not None:
        out["logprob"] = torch.full((n,), 7.0, device="cuda")
    if top:
        out["top_token"] = torch.full((n, top), 77, dtype=torch.int32, device="cuda")
        out["top_logprob"] = torch.full((n, top), 7.0, device="cuda")
    if stream is not None:
        torch.cuda.synchronize()   # (the presets are another stream's work)
    vl.vl_token_logprobs(x, token=token, mask=mask, scale=scale, stream=stream, **out)
    return out


def check_scores(out, want, what=""):
    near(out["stat"], want.stat, want.stat_err, what + " stat")
    near(out["entropy"], want.entropy, want.entropy_err, what + " entropy")
    if "logprob" in out:
        near(out["logprob"], want.logprob, want.logprob_err, what + " logprob")
    if "top_token" in out:
        got = out["top_token"].cpu().numpy()
        assert (got == want.top_token).all(), f"{what} top_token {np.argwhere(got != want.top_token)[:4].tolist()}"
        near(out["top_logprob"], want.top_logprob, want.top_err, what + " top_logprob")


def check_all(x, token=None, mask=None, scale=1.0, top=0, seed=1, what=""):
    """scores, then the gradients from what they wrote: of the log probability, of the entropy, of both"""
    n, v = x.shape
    out = scores(x, token, mask, scale, top)
    want = Rows(x, token, mask, scale, top)
    check_scores(out, want, what)
    gen = torch.Generator().manual_seed(seed)
    g, e = torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    for gg, ee in ((g, None), (None, e), (g, e)):
        if token is None and gg is not None:
            continue
        grad = torch.full((n, v), 7.0, dtype=x.dtype, device="cuda")
        vl.vl_token_logprobs_grad(x, out["stat"], grad, token=token, mask=mask, scale=scale, entropy=out["entropy"],
                                  g_logprob=None if gg is None else gg.cuda(), g_entropy=None if ee is None else ee.cuda())
        d, err = want.grad(x.dtype, gg, ee)
        near(grad, d, err, f"{what} grad g {gg is not None} e {ee is not None}")
    return out, want


def bell(n, v, dtype, seed, width=2.0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((n, v), generator=gen) * width
    x[torch.arange(n), torch.randint(0, v, (n,), generator=gen)] += 6.0
    return x.to(dtype).cuda()


def tokens(n, v, seed):
    return torch.randint(0, v, (n,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


def some_bits(n, v, seed, share=0.5):
    return np.random.default_rng(seed).random((n, v)) < share


SIZES = [1, 2, 3, 7, 8, 9, 63, 64, 65, 255, 257, 511, 512, 513, 777, 1023, 1024, 1025, 2047, 2048, 2049, 4097, 8191, 12288, 16385]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("v", SIZES)
def test_sizes(v, dtype):
    n = 5
    x = bell(n, v, dtype, v)
    check_all(x, tokens(n, v, v), top=min(5, v), what="no mask")
    check_all(x, tokens(n, v, v + 1), mask=words_of(some_bits(n, v, v)).cuda(), scale=0.7, top=32, what="mask")


@pytest.mark.parametrize("n,v,dtype", [(1, 131072, BF16), (2, 131077, F16), (3, 50001, F32), (1, 300000, BF16), (130, 20011, BF16), (700, 4099, F16),
                                       (1, 1 << 20, BF16), (40, 50001, F16)])
def test_long_rows(n, v, dtype):
    """rows shared among workgroups, few and many"""
    x = bell(n, v, dtype, n + v)
    check_all(x, tokens(n, v, 3), top=20, what="no mask")
    check_all(x, tokens(n, v, 4), mask=words_of(some_bits(n, v, 5, 0.3)).cuda(), scale=1.4, top=3, what="mask")


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 300, 1025, 5000])
def test_row_counts(n):
    v = 512
    x = bell(n, v, BF16, n)
    t = tokens(n, v, n)
    t[::7] = -1
    check_all(x, t, mask=words_of(some_bits(n, v, n)).cuda(), top=8)


def test_more_rows_than_a_grid_has_room_for_one_by_one():
    n, v = 300_000, 3
    x = bell(n, v, F32, 1)
    check_all(x, tokens(n, v, 2), top=2)


def odd_rows(v, dtype):
    """(logits, token, allowed, what) of rows where it can go wrong"""
    gen = torch.Generator().manual_seed(v)
    low, inf, nan = torch.finfo(dtype).min, float("inf"), float("nan")
    one = [v // 2]
    base = torch.randn(v, generator=gen)
    rows = []

    def row(x, token, keep=None, what=""):
        bits = np.ones(v, bool) if keep is None else np.zeros(v, bool)
        if keep is not None:
            bits[keep] = True
        rows.append((x, token, bits, what))

    def with_(value, where):
        x = base.clone()
        x[where] = value
        return x
    some = sorted({0, v // 3, v - 1})
    others = [t for t in range(v) if t not in some]
    row(base, 0, [], "mask leaves nothing")
    row(base, one[0], one, "one token left")
    row(base, v - 1, [0] if v > 1 else [], "given token not allowed")
    row(base, v, None, "token past the vocabulary")
    row(base, 2 ** 31 - 1, some, "token far past it")
    row(torch.full((v,), low), v // 2, None, "all the lowest value")
    row(with_(low, some), some[-1], None, "some the lowest value, given one of them")
    row(torch.full((v,), low), 0, some, "some of the lowest")
    row(torch.full((v,), -inf), 0, None, "all -infinity")
    row(torch.full((v,), -inf), 0, some, "allowed ones -infinity")
    row(with_(-inf, some), some[0], None, "given token -infinity")
    row(torch.full((v,), 1.25), v // 2, None, "all equal")
    row(torch.where(torch.arange(v) % 2 == 0, 0.0, -0.0), 0, None, "zeros of both signs")
    row(with_(nan, some), 0, others, "NaN in masked places")
    row(with_(inf, some), others[0] if others else 0, others, "+infinity in masked places")
    row(with_(nan, [v - 1]), 0, None, "NaN")
    row(with_(inf, [v // 2]), 0, None, "+infinity")
    row(with_(inf, [v // 2]), v // 2, None, "+infinity given")
    row(torch.full((v,), nan), -1, None, "padding, NaN")
    row(base, -2 ** 31, [], "padding, nothing allowed")
    row(torch.arange(v).float() / 64, v - 1, None, "ascending")
    row(-torch.arange(v).float() / 64, v - 1, None, "descending")
    row(base * torch.finfo(dtype).max / 16, v // 2, None, "huge")
    row(with_(torch.finfo(dtype).max, one), 0, None, "the largest value")
    row(base * 1e-30, 0, None, "tiny")
    row(with_(60.0, one), one[0], None, "one far above")
    row(with_(60.0, one), 0, None, "given far below")
    return rows


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("v", [1, 2, 9, 70, 512, 513, 2500, 20011])
@pytest.mark.parametrize("scale", [1.0, 0.01, 30.0])
def test_odd_rows(v, dtype, scale):
    rows = odd_rows(v, dtype)
    x = torch.stack([r[0] for r in rows]).to(dtype).cuda()
    t = torch.tensor([r[1] for r in rows], dtype=torch.int32).cuda()
    bits = np.stack([r[2] for r in rows])
    check_all(x, t, mask=words_of(bits).cuda(), scale=scale, top=min(32, v + 2), what=f"{[r[3] for r in rows]}")
    check_all(x, None, mask=words_of(bits).cuda(), scale=scale, top=1, what="no token")
    whole = [k for k, r in enumerate(rows) if r[2].all()]
    check_all(x[whole].contiguous(), t[whole].contiguous(), scale=scale, top=20, what="no mask")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,v", [(3, 512), (3, 515), (2, 9000), (300, 700), (1, 131072), (2, 98304), (2, 70001), (1100, 1040), (2100, 1041)])
@pytest.mark.parametrize("first,after", [(1, 0), (3, 5), (8, 8), (13, 0)])
def test_windows_of_wider_rows(dtype, n, v, first, after):
    """logits and gradient in rows of another pitch and start; what lies beside them stays, and is not looked at"""
    pitch = first + v + after
    full = torch.full((n, pitch), float("nan"), dtype=dtype, device="cuda")
    x = full[:, first:first + v]
    x.copy_(bell(n, v, dtype, 8))
    t = tokens(n, v, 9)
    wide_mask = torch.full((n, (v + 31) // 32 + 3), -1, dtype=torch.int32)
    bits = some_bits(n, v, 10)
    wide_mask[:, :(v + 31) // 32] = words_of(bits)
    if v % 32:   # bits past the vocabulary do not count
        wide_mask[:, v // 32] |= -(1 << (v % 32))
    wide_mask = wide_mask.cuda()
    out, want = check_all(x, t, mask=wide_mask, top=6)
    g, e = torch.randn(n), torch.randn(n)
    side = torch.full((n, pitch + 7), 3.0, dtype=dtype, device="cuda")
    at = (first * 5) % 7
    vl.vl_token_logprobs_grad(x, out["stat"], side[:, at:at + v], token=t, mask=wide_mask, entropy=out["entropy"], g_logprob=g.cuda(), g_entropy=e.cuda())
    d, err = want.grad(dtype, g, e)
    near(side[:, at:at + v], d, err, "gradient in wider rows")
    assert (side[:, :at] == 3.0).all() and (side[:, at + v:] == 3.0).all()
    # in place
    vl.vl_token_logprobs_grad(x, out["stat"], x, token=t, mask=wide_mask, entropy=out["entropy"], g_logprob=g.cuda(), g_entropy=e.cuda())
    near(x, d, err, "gradient in place")
    assert full[:, :first].isnan().all() and full[:, first + v:].isnan().all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("v", [4095, 4096, 4097, 8190, 8191, 8192, 8193, 16384, 2056, 2087])
@pytest.mark.parametrize("masked", [False, True])
def test_gradient_at_the_ends_of_long_rows(v, dtype, masked):
    """rows at odd and even places whose chunks fill pieces to the last one, or one more or less; beside them, in place, and from the other parity"""
    n = 4
    t = torch.tensor([0, v - 1, v // 2, 7], dtype=torch.int32).cuda()
    mask = words_of(some_bits(n, v, 3)).cuda() if masked else None   # (no word more than the row needs)
    for first, pitch in ((0, v + 1), (1, v + 2), (1, v + 1)):
        full = torch.full((n * pitch + first + 9,), 7.0, dtype=dtype, device="cuda")
        x = full.as_strided((n, v), (pitch, 1), first)
        x.copy_(bell(n, v, dtype, v))
        out = scores(x, t, mask)
        want = Rows(x, t, mask)
        g, e = torch.tensor([1.0, -2.0, 0.5, 3.0]), torch.tensor([0.5, 1.0, -1.0, 0.0])
        d, err = want.grad(dtype, g, e)
        args = dict(token=t, mask=mask, entropy=out["entropy"], g_logprob=g.cuda(), g_entropy=e.cuda())
        beside = torch.ones(full.shape, dtype=torch.bool, device="cuda")
        beside.as_strided((n, v), (pitch, 1), first)[:] = False
        for shift in (0, 1):
            side = torch.full_like(full, 7.0)
            to = side.as_strided((n, v), (pitch, 1), first + shift)
            vl.vl_token_logprobs_grad(x, out["stat"], to, **args)
            near(to, d, err, f"start {first}, pitch {pitch}, shift {shift}")
            assert (side[shift:][beside[:len(side) - shift]] == 7.0).all() and (side[:shift] == 7.0).all()
        vl.vl_token_logprobs_grad(x, out["stat"], x, **args)
        near(x, d, err, "in place")
        assert (full[beside] == 7.0).all()


@pytest.mark.parametrize("n,v", [(4, 512), (4, 3001), (1, 70000)])
def test_one_mask_for_all_rows(n, v):
    x, t = bell(n, v, BF16, 3), tokens(n, v, 4)
    bits = some_bits(1, v, 5)
    shared = words_of(bits).cuda()
    check_all(x, t, mask=shared[0], top=4)
    check_all(x, t, mask=shared.expand(n, -1), top=4)


@pytest.mark.parametrize("n,v", [(3, 512), (2, 5000), (1, 131072), (300, 4096)])
@pytest.mark.parametrize("top", [1, 2, 31, 32])
def test_alternatives_among_equal_logits(n, v, top):
    """few different values, so that most places are decided by the token, in rows and in parts of rows"""
    rng = np.random.default_rng(top + v)
    x = torch.from_numpy(rng.integers(0, 3, (n, v)).astype(np.float32)).to(BF16).cuda()
    check_all(x, tokens(n, v, 1), top=top, what="three values")
    x = torch.zeros((n, v), dtype=BF16, device="cuda")
    check_all(x, None, top=top, what="one value")
    x[:, v - top:] = 1.0
    check_all(x, None, top=top, what="the last ones")
    x = torch.arange(v, dtype=F32, device="cuda").repeat(n, 1)
    check_all(x, None, top=top, what="ascending", scale=1e-4)
    # the largest ones side by side, and at one distance from each other
    for step in (1, 8, 64, 512, 2048):
        y = torch.zeros((n, v), dtype=F16, device="cuda")
        y[:, (torch.arange(40) * step) % v] = 2.0
        check_all(y, None, top=top, what=f"distance {step}")


@pytest.mark.parametrize("v,dtype,top", [(1, BF16, 8), (9, F16, 8), (127, BF16, 3), (128, BF16, 8), (250, F16, 4), (512, BF16, 2), (1023, F16, 2), (1024, BF16, 1),
                                         (64, F32, 16), (128, F32, 8), (129, F32, 4), (256, F32, 4), (500, F32, 1)])
def test_few_alternatives_of_many_short_rows(v, dtype, top):
    rows = odd_rows(v, dtype)
    x = torch.stack([r[0] for r in rows]).to(dtype).cuda()
    n = 2048 * top + 13   # (teams of lanes without a row at the end)
    which = torch.arange(n) % len(rows)
    bits = np.stack([r[2] for r in rows])
    t = torch.tensor([r[1] for r in rows], dtype=torch.int32)[which].cuda()
    for mask in (None, words_of(bits)[which].cuda()):
        few = scores(x, None, None if mask is None else words_of(bits).cuda(), top=top)
        check_scores(few, Rows(x, None, None if mask is None else words_of(bits).cuda(), top=top), "few rows")
        out = scores(x[which.cuda()], t, mask, top=top)
        there = t >= 0
        for k in ("top_token", "top_logprob", "stat", "entropy"):   # few rows take another way
            a, b = out[k][there].float(), few[k][which.cuda()][there].float()
            assert torch.allclose(a, b, rtol=2.0 ** -18, atol=2.0 ** -18, equal_nan=True) and (k != "top_token" or (a == b).all()), k
        assert (out["top_token"][~there] == -1).all()
    y = bell(n, v, dtype, top)
    y = (y.float() * 4).round().to(dtype)   # many are equal
    want = y.float().sort(dim=1, descending=True, stable=True).indices[:, :top].int()
    got = scores(y, None, top=top)["top_token"]
    assert (got[:, :min(top, v)] == want).all() and (got[:, v:] == -1).all()


@pytest.mark.parametrize("v,dtype,n", [(1041, BF16, 27), (2500, F32, 300), (1100, F16, 1200), (1033, BF16, 2500), (515, F32, 2100), (20011, BF16, 130), (70001, F16, 20), (33001, F32, 27),
                                       (131073, BF16, 2)])
@pytest.mark.parametrize("first", [0, 1])
def test_one_alternative_of_long_rows(v, dtype, n, first):
    """odd values and equal logits, in rows that start at even and odd places"""
    rows = odd_rows(v, dtype)[-n:]
    which = torch.arange(n) % len(rows)
    small = torch.stack([r[0] for r in rows]).to(dtype)
    x = torch.full((n, v + first + 2), float("nan"), dtype=dtype, device="cuda")[:, first:first + v]
    x.copy_(small[which])
    t = torch.tensor([r[1] for r in rows], dtype=torch.int32)[which].cuda()
    bits = words_of(np.stack([r[2] for r in rows]))
    for mask in (None, bits):
        want = Rows(small, t[:len(rows)], mask, top=1)
        out = scores(x, t, None if mask is None else mask[which].cuda(), top=1)
        for at in range(0, n, len(rows)):   # (rows at odd and even places are summed in chunks of their own: none equals another in its last bits)
            some = min(len(rows), n - at)
            if some < len(rows):
                want = Rows(small[:some], t[:some], None if mask is None else mask[:some], top=1)
            check_scores({k: o[at:at + some] for k, o in out.items()}, want, f"rows from {at} on")


@pytest.mark.parametrize("v", [512, 4096, 32768, 131072, 1 << 20])
@pytest.mark.parametrize("top", [1, 8, 20, 32])
def test_alternatives_that_stand_together(v, top):
    """the best logits of a row in few of the places that are looked at together: 8 tokens in a row, such eights 512 or 2,048 tokens
    apart, and the first 32 tokens of every eighth 4,096"""
    t = torch.arange(v)
    rows = []
    for lanes in (64, 256):
        lane, turn = t // 8 % lanes, t // (8 * lanes)
        rows.append(torch.where(lane < 12, 200 - 8 * lane + turn % 8, 0))   # one lane's all above the next one's
        rows.append(torch.where(lane < 12, 100 + 8 * lane - turn % 8, 0))
    rows.append(torch.where((t // 4096 % 8 == 0) & (t % 4096 < 32), 200 - t % 4096, 0))
    rows.append(-(t // 8) % 200)
    x = torch.stack(rows).float()
    for dtype in (BF16, F32):   # (every value is exact in either)
        for n in (1, len(rows)):
            y = x[:n] if n > 1 else x[4:5]
            out = scores(y.to(dtype).cuda(), None, top=top)
            check_scores(out, Rows(y, None, top=top))


@pytest.mark.parametrize("n,v", [(2048, 131072), (60, 1 << 20), (1, 1 << 24)])
def test_many_equal_terms(n, v):
    """a row's terms are not added up one by one: with 512 logits of x and the others 0, 64 lanes that take 32 at a time and 1,024
    that take 16 make v / 2048 additions in a row at most, and some 50 for the batch and the joining"""
    x = torch.zeros((n, v), dtype=F16, device="cuda")
    x[:, :512] = 0.357
    m = float(x[0, 0])
    s = 512 + (v - 512) * np.exp(-m)
    u = 2.0 ** -24
    sum_err = u * (4 * m + 4 + v / 2048 + 50)
    out = scores(x)
    log_sum, share = np.log(s), (v - 512) * np.exp(-m) / s
    near(out["stat"], np.tile([m, log_sum], (n, 1)), np.tile([0, sum_err + u * (log_sum + 2)], (n, 1)))
    near(out["entropy"], np.full(n, log_sum + m * share), np.full(n, sum_err + m * (2 * sum_err + 12 * u) + 3 * u * log_sum))


def test_outputs_that_are_not_asked_for():
    n, v = 6, 700
    x, t = bell(n, v, F16, 1), tokens(n, v, 2)
    want = Rows(x, t, top=3)
    one = torch.full((n,), 7.0, device="cuda")
    vl.vl_token_logprobs(x, token=t, logprob=one)
    near(one, want.logprob, want.logprob_err)
    vl.vl_token_logprobs(x, entropy=one)
    near(one, want.entropy, want.entropy_err)
    k = torch.full((n, 3), 7, dtype=torch.int32, device="cuda")
    vl.vl_token_logprobs(x, top_token=k)
    assert (k.cpu().numpy() == want.top_token).all()
    lq = torch.full((n, 3), 7.0, device="cuda")
    vl.vl_token_logprobs(x, top_logprob=lq)
    near(lq, want.top_logprob, want.top_err)


@pytest.mark.parametrize("dtype", [F32])
def test_gradient_against_differences(dtype):
    """of the kernel's own numbers, where 32 bits allow it: the step h = 2^-6 leaves h^2 times a third derivative (at most 1 for
    the log probability, 8 for the entropy of so few tokens), the numbers' roundings 2^-22 / h each"""
    n, v, h = 3, 7, 2.0 ** -6
    x = torch.randn((n, v), generator=torch.Generator().manual_seed(4)).cuda()
    t = tokens(n, v, 5)
    g, e = torch.tensor([1.0, -2.0, 0.5]).cuda(), torch.tensor([0.5, 1.0, -1.0]).cuda()
    out = scores(x, t)
    grad = torch.empty_like(x)
    vl.vl_token_logprobs_grad(x, out["stat"], grad, token=t, entropy=out["entropy"], g_logprob=g, g_entropy=e)
    for k in range(v):
        up, down = x.clone(), x.clone()
        up[:, k] += h
        down[:, k] -= h
        a, b = scores(up, t), scores(down, t)
        diff = (g * (a["logprob"] - b["logprob"]) + e * (a["entropy"] - b["entropy"])) / (2 * h)
        assert (diff - grad[:, k]).abs().max().item() < 20 * h * h + 8 * 2.0 ** -22 / h


def test_rows_far_apart():
    """a row that starts past 4 GB and 2^31 elements"""
    v, n = 1000, 3
    pitch = (1 << 30) + 8
    full = torch.empty(2 * pitch + v, dtype=BF16, device="cuda")
    x = full.as_strided((n, v), (pitch, 1))
    x.copy_(bell(n, v, BF16, 1))
    out, want = check_all(x, tokens(n, v, 2), top=4)
    g = torch.randn(n)
    vl.vl_token_logprobs_grad(x, out["stat"], x, token=tokens(n, v, 2), g_logprob=g.cuda())
    d, err = want.grad(BF16, g)
    near(x, d, err)


def test_two_streams_and_a_recorded_pass():
    """calls on two streams at once, then a pass recorded with memory of its own and replayed among eager calls"""
    n, v = 4, 131072
    xs = [bell(n, v, BF16, k) for k in range(2)]
    ts = [tokens(n, v, k) for k in range(2)]
    wants = [Rows(x, t, top=8) for x, t in zip(xs, ts)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()

    def room():
        return dict(logprob=torch.full((n,), 7.0, device="cuda"), entropy=torch.full((n,), 7.0, device="cuda"), stat=torch.full((n, 2), 7.0, device="cuda"),
                    top_token=torch.full((n, 8), 77, dtype=torch.int32, device="cuda"), top_logprob=torch.full((n, 8), 7.0, device="cuda"))
    outs = [[room() for _ in range(6)] for _ in range(2)]
    torch.cuda.synchronize()
    for turn in range(6):
        for k in range(2):
            vl.vl_token_logprobs(xs[k], token=ts[k], stream=streams[k], **outs[k][turn])
    torch.cuda.synchronize()
    for k in range(2):
        for o in outs[k]:
            check_scores(o, wants[k])
    x, t = xs[0].clone(), ts[0].clone()
    out = dict(logprob=torch.zeros(n, device="cuda"), entropy=torch.zeros(n, device="cuda"), stat=torch.zeros((n, 2), device="cuda"),
               top_token=torch.zeros((n, 8), dtype=torch.int32, device="cuda"), top_logprob=torch.zeros((n, 8), device="cuda"))
    grad, g = torch.zeros_like(x), torch.randn(n)
    g_dev = g.cuda()

    def one_pass():
        vl.vl_token_logprobs(x, token=t, **out)
        vl.vl_token_logprobs_grad(x, out["stat"], grad, token=t, g_logprob=g_dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one_pass()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one_pass()
    for k in (1, 0, 1, 1):
        x.copy_(xs[k])
        t.copy_(ts[k])
        grad.zero_()
        graph.replay()
        eager = scores(xs[1 - k], ts[1 - k], top=8)
        torch.cuda.synchronize()
        check_scores(out, wants[k], "replayed")
        check_scores(eager, wants[1 - k], "eager")
        d, err = wants[k].grad(BF16, g)
        near(grad, d, err, "replayed gradient")


@pytest.mark.parametrize("n,v,top", [(1, 131072, 20), (300, 20011, 5), (3000, 512, 8), (2500, 4097, 0), (700, 300, 0)])
def test_equal_calls_give_equal_bits(n, v, top):
    x, t = bell(n, v, BF16, 1), tokens(n, v, 2)
    first = scores(x, t, top=top)
    g = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda()
    grads = []
    for _ in range(4):
        again = scores(x, t, top=top)
        for name in first:
            assert torch.equal(first[name], again[name]), name
        grads.append(torch.empty_like(x))
        vl.vl_token_logprobs_grad(x, again["stat"], grads[-1], token=t, entropy=again["entropy"], g_logprob=g, g_entropy=g)
    assert all(torch.equal(grads[0], y) for y in grads)


def test_refusals_of_the_binding():
    x = torch.zeros((4, 64), device="cuda")
    out = torch.zeros(4, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")

    def code(*args, **named):
        with pytest.raises(vl.VlError) as err:
            vl.vl_token_logprobs(*args, **named)
        return err.value.code
    assert code(x, entropy=out.cpu()) == -7
    assert code(x, token=t.cpu(), logprob=out) == -7
    assert code(x, mask=torch.zeros((4, 2), dtype=torch.int32), entropy=out) == -7
    assert code(x.double(), entropy=out) == -3
    assert code(x, entropy=out.half()) == -3
    assert code(x, token=t.long(), logprob=out) == -3
    assert code(x.t(), entropy=out) == -2                        # rows that are not contiguous
    assert code(x[0], entropy=out) == -2
    assert code(x, entropy=out[:3]) == -2
    assert code(x, entropy=torch.zeros(8, device="cuda")[::2]) == -2
    assert code(x, mask=torch.zeros((4, 1), dtype=torch.int32, device="cuda"), entropy=out) == -2
    assert code(x[:1].expand(4, 64), entropy=out) == -2          # rows of no pitch
    assert code(x, token=t) == -1 and code(x, logprob=out) == -1
    assert code(x, entropy=out, scale=0.0) == -3 and code(x, entropy=out, scale=1e300) == -3
    assert code(x[:0], entropy=out[:0]) == -2 and code(x[:, :0], entropy=out) == -3
    assert code(x, top_token=torch.zeros((4, 33), dtype=torch.int32, device="cuda")) == -3
    stat = torch.zeros((4, 2), device="cuda")
    for grad, want in ((torch.zeros((4, 63), device="cuda"), -2), (x.half(), -3), (x.cpu(), -7), (None, -1)):
        with pytest.raises(vl.VlError) as err:
            vl.vl_token_logprobs_grad(x, stat, grad, token=t, g_logprob=out)
        assert err.value.code == want
    torch.cuda.synchronize()
    assert (out == 0).all()


def test_forms_of_a_stream():
    """a torch stream, its handle as a number, the default stream as None and as 0, a ctypes pointer"""
    import ctypes
    x, t = bell(2, 131072, BF16, 1), tokens(2, 131072, 2)
    want = Rows(x, t, top=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, 0, torch.cuda.current_stream(), side, side.cuda_stream, ctypes.c_void_p(side.cuda_stream), ctypes.c_void_p(0)):
        out = scores(x, t, top=4, stream=stream)
        torch.cuda.synchronize()
        check_scores(out, want, str(stream))


def test_work_of_the_callers():
    x, t = bell(1, 131072, BF16, 1), tokens(1, 131072, 1)
    lp = torch.zeros(1, device="cuda")
    need = vl.vl_token_logprobs_work(x, token=t, logprob=lp)
    want = Rows(x, t)
    work = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        vl.vl_token_logprobs(x, token=t, logprob=lp, work=work[:need] if need else None)
        near(lp, want.logprob, want.logprob_err)
    assert (work[need:] == 255).all()
    if need:
        with pytest.raises(vl.VlError) as err:
            vl.vl_token_logprobs(x, token=t, logprob=lp, work=work[:need - 1])
        assert err.value.code == -2
