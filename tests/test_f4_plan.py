"""How products with both operands in 4-bit floating point are cut: the cases that the GPU tests multiply take every path of the kernels."""
import numpy as np
import pytest

# M, K, N and the plan on a B200 (148 multiprocessors, 33 clusters of four and 15 of eight CTAs at once): rows of a tile, shares of k, rounds of the 74
# pairs, rows numbered first, output past L2
PROMPTS = [
    (130, 256, 12002, 64, 1, 2, 1, 0), (100, 256, 19001, 64, 1, 3, 1, 0), (130, 96, 19001, 64, 1, 4, 1, 0), (330, 288, 12001, 128, 1, 2, 1, 0),
    (330, 256, 19001, 128, 1, 4, 1, 0), (100, 800, 19001, 128, 1, 2, 0, 0), (520, 288, 9002, 192, 1, 2, 1, 0), (520, 256, 19001, 192, 1, 4, 1, 0),
    (2500, 288, 2040, 192, 1, 2, 0, 0), (130, 2080, 19001, 192, 1, 2, 0, 0), (450, 288, 9001, 256, 1, 1, 0, 0), (777, 2080, 9002, 256, 1, 2, 1, 0),
    (1000, 96, 19001, 256, 1, 5, 1, 0), (1300, 256, 9001, 256, 1, 3, 1, 0), (777, 3584, 4608, 256, 1, 1, 0, 0), (1800, 288, 18944, 256, 1, 8, 1, 1),
    (1801, 96, 19001, 192, 1, 11, 1, 1)]
SHARES = [(65, 4096, 264, 64, 4), (100, 8256, 4100, 128, 2), (100, 4096, 2600, 128, 4), (129, 14336, 4100, 192, 2), (520, 8256, 2600, 192, 2), (520, 8256, 1000, 192, 4),
          (129, 8256, 2601, 192, 4), (250, 14336, 4100, 256, 2), (250, 8256, 2600, 256, 4)]


@pytest.fixture(scope="module")
def B():
    from paper_2511_11248_b200 import build, binding
    build.build()
    return binding


def rounds(p):
    return -(-p["tiles_m"] * p["tiles_n"] // 74)


@pytest.mark.parametrize("block", [32, 16])
def test_the_cases_take_every_path(B, block):
    seen = set()
    for M, K, N, rows, shares, n, first, past in PROMPTS:
        p = B.tman_debug_f4_plan_for(1, M, K, N, block, 148, 33, 15)
        assert (p["pair"], p["rows"], p["shares"], rounds(p), p["flags"] & 1, p["flags"] >> 1) == (1, rows, shares, n, first, past), (M, K, N, p)
        assert p["workers"] == min(74, p["tiles_m"] * p["tiles_n"]) and p["tiles_m"] == -(-M // rows) and p["tiles_n"] == -(-N // 256)
        seen.add((rows, min(n, 3)))
    for M, K, N, rows, shares in SHARES:
        p = B.tman_debug_f4_plan_for(1, M, K, N, block, 148, 33, 15)
        assert (p["pair"], p["rows"], p["shares"]) == (1, rows, shares), (M, K, N, p)
        assert p["workers"] == shares * p["tiles_m"] * p["tiles_n"] and p["tiles_m"] * p["tiles_n"] <= (33 if shares == 2 else 15)
        seen.add((rows, -shares))
    assert seen >= {(r, n) for r in (64, 128, 192, 256) for n in (2, 3)} - {(64, 2)} and seen >= {(r, -s) for r in (128, 192, 256) for s in (2, 4)} | {(64, -4)}


def test_no_more_clusters_than_the_device_holds(B):
    rng = np.random.default_rng(0)
    for _ in range(400):
        M, K, N = int(2 ** rng.uniform(6, 11)), int(2 ** rng.uniform(1, 9)) * 32, int(2 ** rng.uniform(5, 14))
        held = [int(rng.integers(0, 38)), int(rng.integers(0, 19))]
        p = B.tman_debug_f4_plan_for(1, M, K, N, 32, 148, *held)
        tiles = p["tiles_m"] * p["tiles_n"]
        if p["pair"] and p["shares"] > 1:
            assert tiles <= held[p["shares"] // 4] and p["workers"] == p["shares"] * tiles
            assert -(-K // 256) >= 2 * p["shares"]
        elif not p["pair"]:
            assert p["shares"] <= 8 and p["tiles_n"] * p["shares"] <= max(148, p["tiles_n"]) and p["stages"] >= 1
            assert p["shares"] < 3 or p["tiles_n"] <= (held[0] * 4 // p["shares"] if p["shares"] < 7 else held[1])


def test_refusals(B):
    for over, status in ((dict(M=0), 2), (dict(K=48), 2), (dict(N=0), 2), (dict(block=64), 2), (dict(op=2), 3), (dict(op=0), 2), (dict(sms=1), 2), (dict(four=-1), 2)):
        a = dict(op=1, M=100, K=256, N=512, block=32, sms=148, four=33, eight=15, **{})
        a.update(over)
        with pytest.raises(B.TmanError) as e:
            B.tman_debug_f4_plan_for(*a.values())
        assert e.value.status == status, over
    assert B.lib().tman_debug_f4_plan_for(1, 100, 256, 512, 32, 148, 33, 15, None) == 1 and B.lib().tman_debug_f4_plan(1, 100, 256, 512, 32, None) == 1


# K, N, rows from which pairs of CTAs were measured to be faster by a twentieth and more, rows up to which streams of weights were; of either block
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("K,N,pairs,streams", [(4096, 1024, 0, 48), (4096, 4096, 64, 48), (2048, 2048, 48, 24), (2048, 8192, 32, 16), (3584, 4608, 48, 24), (14336, 4096, 0, 56),
                                               (18944, 3584, 48, 24), (18944, 512, 0, 64), (8192, 8192, 40, 24), (28672, 8192, 40, 16), (8192, 3584, 56, 40), (4096, 14336, 0, 32),
                                               (28672, 1024, 0, 64), (512, 512, 44, 16), (7168, 7168, 40, 24)])
def test_few_rows_go_to_the_faster_kernel(B, K, N, pairs, streams, block):
    for M in range(1, 66):
        p = B.tman_debug_f4_plan_for(1, M, K, N, block, 148, 33, 15)["pair"]
        assert not (p and M <= streams) and not (pairs and M >= pairs and not p), M


@pytest.mark.parametrize("block", [32, 16])
def test_a_ring_has_three_stages_or_all_that_its_share_takes(B, block):
    """Also where the sums of the shares, which lie behind it, take a third of half an SM's memory."""
    for M in range(1, 65):
        for K, N in ((14336, 4096), (4096, 4096), (28672, 4096), (18944, 512), (4096, 14336), (2048, 512), (96, 40)):
            for op in (0, 1):
                if op == 0 and M > 8:
                    continue
                p = B.tman_debug_f4_plan_for(op, M, K, N, block, 148, 33, 15)
                if not p["pair"]:
                    assert p["stages"] >= min(3, -(-K // 256 // p["shares"])), (op, M, K, N, p)
