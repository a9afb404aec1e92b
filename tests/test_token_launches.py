"""The token operators' host code on a stand-in runtime: what they launch, and that they do nothing else."""
import ctypes as C
import random

from stand_in import in_own_process

P = 1 << 20   # a pointer that nothing follows


def _scores(s, n, v, kind, top, mask=True, ld=None, odd=0, stream=0x77):
    """(launches, work bytes) of one call"""
    from paper_2506_17506_amd import binding as b
    lib = s.vl.load()
    rows = b._TokenRows(P + odd, ld or v, P if mask else None, (v + 31) // 32 if mask else 0, P, n, v, kind, 1.0)
    out = b._TokenScores(P, P, P, P if top else None, P if top else None, top, 0)
    need = C.c_uint64()
    assert lib.vl_token_logprobs_work(C.byref(rows), C.byref(out), C.byref(need)) == 0
    s.launches.clear()
    assert lib.vl_token_logprobs(C.byref(rows), C.byref(out), P if need.value else None, need.value, stream) == 0
    return list(s.launches), need.value


@in_own_process
def test_scores_launch_kernels_only_and_cover_their_rows(s):
    rng = random.Random(5)
    before = s.counts()
    sizes = [(1, 1), (1, 131072), (1, 1 << 24), (47, 70000), (48, 70000), (127, 1 << 20), (128, 50001), (1023, 8), (1024, 9000), (2047, 300000), (2048, 131072), (70000, 4099),
             (2 ** 31 - 1, 3), (2 ** 31 - 1, 1040)]
    sizes += [(int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 18))) for _ in range(200)]
    for n, v in sizes:
        for kind in (0, 1, 2):
            top = rng.choice([0, 0, 1, 20, 32])
            ld = v + rng.choice([0, 0, 1, 64])
            launches, need = _scores(s, n, v, kind, top, mask=rng.random() < 0.5, ld=ld, odd=0 if kind == 0 else rng.choice([0, 0, 2]))
            other = _scores(s, n, v, kind, top, ld=v + 1, odd=0 if kind == 0 else 2)[1]
            assert need == other, (n, v, kind, top, need, other)
            assert 1 <= len(launches) <= 2 and all(x[4] == 0x77 for x in launches)
            for name, grid, block, lds, stream, words in launches:
                assert all(1 <= g for g in grid) and grid[0] * block < 2 ** 32 and grid[1] <= 65535 and grid[2] == 1, (n, v, kind, name, grid)
            name, grid, block = launches[0][:3]
            if "k_scores_long" in name:
                assert grid[1] == min(n, 65535)
                parts = grid[0]
                assert (parts > 1) == (len(launches) == 2) and parts <= 256, (n, v, grid)
                least = n * parts * (16 + 8 * top) if parts > 1 else 0
                assert least <= need <= n * 256 * (16 + 8 * top), (n, v, need, grid)   # (it does not go by where the rows start)
                if parts > 1:
                    assert "k_scores_join" in launches[1][0] and launches[1][1][0] == n and launches[1][2] == 256
            else:
                assert need == 0 and len(launches) == 1 and grid[0] <= 1 << 20
    assert s.counts() == before   # no allocation, no copy, no wait


@in_own_process
def test_the_others_launch_kernels_only(s):
    from paper_2506_17506_amd import binding as b
    lib = s.vl.load()
    before = s.counts()
    rng = random.Random(6)
    for n, v in [(1, 1), (3, 512), (8192, 131072), (70000, 5000), (2 ** 31 - 1, 7)] + [(int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 18))) for _ in range(100)]:
        for kind in (0, 1, 2):
            rows = b._TokenRows(P, v, None, 0, P, n, v, kind, 1.0)
            s.launches.clear()
            assert lib.vl_token_logprobs_grad(C.byref(rows), P, P, P, P, P, v, 0x77) == 0
            (name, grid, block, lds, stream, words), = s.launches
            assert stream == 0x77 and grid[0] * block < 2 ** 32 and grid[1] <= 65535
            if "k_grad_long" in name:
                assert grid[1] == min(n, 65535) and grid[0] * 1024 * (4 if kind == 0 else 8) >= v
    for n, groups in [(1, 1), (100, 1), (256000, 256), (2 ** 31 - 1, 1), (2 ** 31 - 1, 2 ** 31 - 1), (5, 70000)]:
        s.launches.clear()
        w = b._RewardWeights(1, 2, 3, 4)
        assert lib.vl_group_advantages(P, P, n, P, groups, C.byref(w), 1e-6, P, P, 0x77) == 0
        (name, grid, block, lds, stream, words), = s.launches
        assert 1 <= grid[0] <= 65536 and block in (256, 1024)
    for n, m, longest in [(1, 1, 0), (1, 1, 1), (10 ** 9, 1600, 57000), (10 ** 12, 2 ** 31 - 1, 2 ** 32 - 1), (10 ** 9, 1, 10 ** 9), (70000, 70000, 1)]:
        batch = b._PolicyBatch(P, P, P, n, P, P, P, P, m, longest, -0.2, 0.2, 0.1, 0)
        need = C.c_uint64()
        assert lib.vl_policy_loss_work(C.byref(batch), C.byref(need)) == 0
        s.launches.clear()
        assert lib.vl_policy_loss(C.byref(batch), P, P, P if need.value else None, need.value, 0x77) == 0
        first, rest = s.launches[0], s.launches[1:]
        blocks = first[1][0]
        assert 1 <= blocks <= 8192 and need.value == (blocks * 32 if blocks > 1 else 0) and [x[1][0] for x in rest] == [1] * (blocks > 1)
        if need.value:
            s.launches.clear()
            assert lib.vl_policy_loss(C.byref(batch), P, P, P, need.value - 1, 0x77) == -2 and not s.launches
    assert s.counts() == before
