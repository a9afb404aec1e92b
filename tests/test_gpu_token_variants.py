"""The token operators in every way that the sizes choose, for every type, on the GPU: short rows in teams of lanes, long ones by
64, 256 and 1,024 threads, logits beyond the sizes from which they are read past the caches, and more rows than a launch has
workgroups for, so that one takes several.  Many rows are copies of few, which keeps the
definitions in 64 bits (token_reference.py) cheap; an odd number of different rows in rows of odd pitch, so that
each of them stands at even and at odd places."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2506_17506_amd as vl  # noqa: E402
from test_gpu_token_scores import bell, odd_rows, some_bits, tokens  # noqa: E402
from token_reference import Rows, words_of  # noqa: E402

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vl.load()
    yield
    torch.cuda.empty_cache()


class Copies:
    """n rows in turn of few different ones: with odd values and masks if `odd`, and a bell's"""

    def __init__(self, n, v, dtype, masked, odd, pitch=None, few=9):
        small, token, bits = bell(few, v, dtype, v), tokens(few, v, v + 1), some_bits(few, v, v + 2, 0.6)
        if odd:
            rows = odd_rows(v, dtype)
            rows = rows[:len(rows) - (len(rows) + few + 1) % 2]   # (an odd number in all)
            small = torch.cat([small, torch.stack([r[0] for r in rows]).to(dtype).cuda()])
            token = torch.cat([token, torch.tensor([r[1] for r in rows], dtype=torch.int32).cuda()])
            bits = np.concatenate([bits, np.stack([r[2] for r in rows])])
        token[3] = -1
        self.few = few = len(small)
        assert few % 2 == 1
        self.which = torch.arange(n, device="cuda") % few
        pitch = pitch or v
        full = torch.full((n, pitch), 7.0, dtype=dtype, device="cuda")
        self.full, self.x = full, full[:, :v]
        for r in range(0, n, 1 << 14):
            self.x[r:r + (1 << 14)] = small[self.which[r:r + (1 << 14)]]
        words = words_of(bits).cuda() if masked else None
        self.token, self.mask = token[self.which], None if words is None else words[self.which]
        self.small = (small, token, words)

    def near(self, got, want, err, what):
        """every copy's rows against one of them; a bounded piece at a time"""
        want = np.where(np.abs(want) > 3.4028236e38, np.copysign(np.inf, want), want)   # what 32 bits do not hold
        want, err = torch.from_numpy(want).cuda(), torch.from_numpy(np.broadcast_to(err, want.shape).copy()).cuda()
        for k in range(self.few):
            w, e, mine = want[k], err[k], got[k::self.few]
            for r in range(0, len(mine), 1 << 10):
                g = mine[r:r + (1 << 10)].double()
                fine = (g == w) | (g.isnan() & w.isnan()) | (w.isfinite() & ((g - w).abs() <= e))
                assert fine.all(), f"{what}: row {k + (r + int((~fine).nonzero()[0, 0])) * self.few}, a copy of {k}: {(~fine).nonzero()[:4].tolist()}"


def check_scores(n, v, dtype, masked, top, odd=False, pitch=None):
    c = Copies(n, v, dtype, masked, odd, pitch)
    small, token, words = c.small
    want = Rows(small, token, words, top=top)
    out = dict(logprob=torch.full((n,), 7.0, device="cuda"), entropy=torch.full((n,), 7.0, device="cuda"), stat=torch.full((n, 2), 7.0, device="cuda"))
    if top:
        out["top_token"] = torch.full((n, top), 77, dtype=torch.int32, device="cuda")
        out["top_logprob"] = torch.full((n, top), 7.0, device="cuda")
    vl.vl_token_logprobs(c.x, token=c.token, mask=c.mask, **out)
    c.near(out["stat"], want.stat, want.stat_err, "stat")
    c.near(out["entropy"][:, None], want.entropy[:, None], want.entropy_err[:, None], "entropy")
    c.near(out["logprob"][:, None], want.logprob[:, None], want.logprob_err[:, None], "logprob")
    if top:
        c.near(out["top_token"], want.top_token.astype(float), 0.0, "top_token")
        c.near(out["top_logprob"], want.top_logprob, want.top_err, "top_logprob")


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("chunks", [1, 16, 17, 32, 33, 64, 65, 128])   # (of 16 bytes)
@pytest.mark.parametrize("masked", [False, True])
def test_short_rows_by_few_lanes(chunks, dtype, masked):
    for v in (chunks * 16 * 8 // torch.finfo(dtype).bits, chunks * 16 * 8 // torch.finfo(dtype).bits - 1):
        for top in (0, 1):
            check_scores(1201, v, dtype, masked, top, odd=True, pitch=v + 1 - v % 2 + 2)


# 16-byte chunks of a row: 1,024 threads each where there are 96 to 512 of them, up to 256 with a compute unit of their own
@pytest.mark.parametrize("n", [150, 301])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("top", [0, 1, 5])
@pytest.mark.parametrize("masked", [False, True])
def test_a_row_by_many_threads(n, dtype, masked, top):
    check_scores(n, 70001 if dtype != F32 else 35001, dtype, masked, top)


# more than 256 MB of logits, by what the rows' number and length choose: a wavefront, 256 threads, 1,024 threads per row
@pytest.mark.parametrize("n,v", [(2101, 65001), (1501, 90001), (401, 340001), (2101, 70001)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("top", [0, 1, 5])
@pytest.mark.parametrize("masked", [False, True])
def test_scores_of_logits_beyond_the_caches(n, v, dtype, masked, top):
    v = v if dtype != F32 else v // 4 * 2 + 1
    assert n * v * torch.finfo(dtype).bits // 8 > 256 << 20
    check_scores(n, v, dtype, masked, top)


@pytest.mark.parametrize("n,v,dtype", [(2101, 65001, F16), (1501, 46001, F32)])
@pytest.mark.parametrize("top", [1, 32])
def test_odd_rows_beyond_the_caches(n, v, dtype, top):
    check_scores(n, v, dtype, True, top, odd=True)


# 65,535 workgroups at most, so that some take two rows; below and beyond 256 MB
@pytest.mark.parametrize("n,v,dtype", [(70001, 1101, BF16), (70001, 1101, F16), (70001, 701, F32), (70001, 2101, BF16), (70001, 1101, F32)])
@pytest.mark.parametrize("top", [0, 1, 5])
@pytest.mark.parametrize("masked", [False, True])
def test_scores_of_more_rows_than_workgroups(n, v, dtype, masked, top):
    check_scores(n, v, dtype, masked, top, odd=True)


def test_more_long_rows_than_workgroups_with_alternatives():
    """256 threads per row (9 GB of logits)"""
    check_scores(65600, 65561, BF16, True, 5)


@pytest.mark.parametrize("n,v,dtype,pitch", [(701, 50001, F32, None), (1401, 50001, BF16, None), (1401, 50001, F16, 50011), (1401, 50000, BF16, None), (70001, 2101, BF16, None),
                                             (70001, 2101, F16, 2111), (70001, 1101, F32, None), (66001, 4201, BF16, None),
                                             (40001, 4201, F16, None), (20001, 3501, F32, None)])
@pytest.mark.parametrize("masked", [False, True])
def test_gradients_beyond_the_caches(n, v, dtype, pitch, masked):
    """logits and gradient more than 256 MB, and rows for which there are not workgroups enough; beside the logits, in place, and from the
    other parity"""
    assert 2 * n * v * torch.finfo(dtype).bits // 8 > 256 << 20
    c = Copies(n, v, dtype, masked, False, pitch)
    small, token, words = c.small
    want = Rows(small, token, words)
    gen = torch.Generator().manual_seed(n)
    g, e = torch.randn(c.few, generator=gen), torch.randn(c.few, generator=gen)
    d, err = want.grad(dtype, g, e)
    stat, entropy = torch.empty((n, 2), device="cuda"), torch.empty(n, device="cuda")
    vl.vl_token_logprobs(c.x, token=c.token, mask=c.mask, stat=stat, entropy=entropy)
    args = dict(token=c.token, mask=c.mask, entropy=entropy, g_logprob=g.cuda()[c.which], g_entropy=e.cuda()[c.which])
    side = torch.full((n, v + 3), 7.0, dtype=dtype, device="cuda")
    for first in (0, 1):
        side.fill_(7.0)
        to = side[:, first:first + v]
        vl.vl_token_logprobs_grad(c.x, stat, to, **args)
        c.near(to, d, err, f"beside, from place {first}")
        assert (side[:, :first] == 7.0).all() and (side[:, first + v:] == 7.0).all()
    vl.vl_token_logprobs_grad(c.x, stat, c.x, **args)
    c.near(c.x, d, err, "in place")
    assert (c.full[:, v:] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("masked", [False, True])
def test_gradients_of_many_rows_that_a_wavefront_holds(dtype, masked):
    """129 to 256 chunks of 16 bytes, by four per lane"""
    v = 1531 if dtype != F32 else 765
    c = Copies(2301, v, dtype, masked, True)
    small, token, words = c.small
    want = Rows(small, token, words)
    e = torch.randn(c.few, generator=torch.Generator().manual_seed(1))
    d, err = want.grad(dtype, None, e)
    stat, entropy = torch.empty((2301, 2), device="cuda"), torch.empty(2301, device="cuda")
    vl.vl_token_logprobs(c.x, token=c.token, mask=c.mask, stat=stat, entropy=entropy)
    vl.vl_token_logprobs_grad(c.x, stat, c.x, token=c.token, mask=c.mask, entropy=entropy, g_entropy=e.cuda()[c.which])
    c.near(c.x, d, err, "in place")
