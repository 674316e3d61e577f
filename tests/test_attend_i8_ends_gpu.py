"""Attention over the 8-bit cache at the ends of what it takes: pages that stand for NaN, windows and lengths next to 2^31, values of any size."""
import numpy as np
import pytest
import torch

from i8_common import TYPES, Sequences, f64, rows_on_device, up, within, workspace
from oracle import i8_oracle as io
from paper_2511_11248_b200 import binding as B, helpers as H
from test_attend_i8_gpu import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("page,lens,new,at,bad", [(16, [34, 9], [4, 1], 33, np.inf), (16, [50, 33], [3, 2], 40, -np.inf), (64, [130, 20], [5, 3], 129, np.nan),
                                                  (16, [120, 40], [100, 40], 70, np.inf), (64, [333, 64], [300, 1], 200, np.nan),
                                                  (16, [333, 70], [300, 70], 332, np.inf), (128, [700, 3], [290, 3], 600, -np.inf)])
def test_a_value_page_that_is_no_number_is_seen_by_the_rows_that_see_it_only(page, lens, new, at, bad, ty):
    """The bad value is in the middle of the new tokens, so that rows in front of its page and, with a window, behind it share a tile with rows that see
    it; in one of two key heads, and then a bad key of another page too."""
    rng = np.random.default_rng(at)
    for keys in (False, True):
        q = Sequences(io, lens, page, 2, 64, rng)
        k, v = rng.standard_normal((sum(lens), 128)), rng.standard_normal((sum(lens), 128))
        v[at, 70] = bad                                   # head 1
        if keys:
            k[at - page if at >= page else at, 3] = bad   # head 0
        q.append(lens, lens, ty, rng, k=k, v=v)
        for window in (0, 1, 2, 20, 100):
            attend(q, lens, new, 4, ty, rng, window=window)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 31 - 90])
def test_windows_next_to_the_largest_number(window):
    """Such a window is none, also for rows in front of the first token, whose positions are negative."""
    rng = np.random.default_rng(12)
    lens = [3, 20, 0, 129]
    for heads in (1, 2):
        q = Sequences(io, lens, 16, 1, 64, rng)
        q.append(lens, lens, "f16", rng)
        attend(q, lens, [5, 2, 1, 3], heads, "f16", rng, window=window)
        attend(q, lens, [5, 30, 0, 10], heads, "f16", rng, window=window)
        attend(q, lens, [100, 70, 70, 129], heads, "f16", rng, window=window)
        attend(q, lens, [300, 2, 70, 64], heads, "f16", rng, window=window)


def test_as_many_steps_as_a_call_may_have():
    """49 for each head of an empty sequence: 43 less than 2^31, so that a sum with the number of multiprocessors is beyond it."""
    S, heads, width = 788, 55617, 64
    assert 2 ** 31 - 148 < S * heads * 49 < 2 ** 31
    row = heads * width
    q, y = torch.zeros(S, row, dtype=torch.float16, device="cuda"), torch.full((S, row), float("nan"), dtype=torch.float16, device="cuda")
    cache = torch.zeros(B.tman_cache_bytes_i8(1, 16, heads, width), dtype=torch.uint8, device="cuda")
    table, lens = torch.zeros(S, 1, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    ws = workspace(B.tman_workspace_bytes_attend(width))
    B.tman_attend_i8(q, row, y, row, B.DTYPE_F16, heads, cache, 1, 16, heads, width, table, 1, lens, None, S, S, 0.125, 0, ws)
    assert B.tman_read_status(ws) == 0
    assert bool((y == 0).all())


@pytest.mark.parametrize("page,n,new,width", [(16, 300, 300, 64), (64, 900, 100, 128), (32, 700, 200, 192), (16, 500, 70, 256)])
def test_prompts_over_equal_values_are_those(page, n, new, width):
    """All tokens have the same value, so every row is that, whatever its probabilities: as long as the row's sum is that of the probabilities that were multiplied.
    In 32 bits: sums of n / 16 tiles and 64 parts, 2^-23 each, and four roundings more; then fp16's own."""
    rng = np.random.default_rng(n)
    q = Sequences(io, [n], page, 1, width, rng)
    v = np.tile(rng.uniform(0.5, 1.0, (1, width)) * rng.choice([-1.0, 1.0], (1, width)), (n, 1))
    q.append([n], [n], "f16", rng, v=v)
    _, held = q.oracle.tokens(0, q.table, n)
    for scale in (0.02, 0.3, 1.0):
        xd, _ = rows_on_device(rng.standard_normal((new, width)), width, torch.float16)
        y = H.alloc_matrix(new, width, torch.float16)
        B.tman_attend_i8(xd, width, y, width, B.DTYPE_F16, 1, q.cache, *q.geometry(), q.table_d, q.table.shape[1], up(np.array([n], dtype=np.int32)),
                         up(np.array([0, new], dtype=np.int32)), 1, new, scale, 0, q.ws)
        assert B.tman_read_status(q.ws) == 0
        ref = np.tile(held[0, 0], (new, 1))
        within(f64(y), ref, (2.0 ** -11 + (n / 16 + 68) * 2.0 ** -23) * np.abs(ref))


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("small", [2.0 ** -2, 2.0 ** -4, 2.0 ** -12, 2.0 ** -19])
def test_prompts_that_look_at_pages_of_small_values(small, ty):
    """Most of each row's probability lies on tokens of values that are small beside the others': what is left of those is right all the same."""
    rng = np.random.default_rng(23)
    n = 420
    q = Sequences(io, [n], 16, 1, 64, rng)
    k, v = rng.standard_normal((n, 64)) * 0.2, rng.standard_normal((n, 64))
    for a in (0, 128, 224):
        k[a:a + 16] += 1.0
        v[a:a + 16] *= small
    q.append([n], [n], ty, rng, k=k, v=v)
    for size in (0.1, 0.4):
        x = np.abs(rng.standard_normal((202, 64))) * size
        attend(q, [n], [200], 1, ty, rng, q16=x, scale=0.5)


def check_small(q, lens, new, heads, ty, rng, window=0):
    """Like `attend`, with bf16's least number in place of fp16's: outputs are small."""
    tt, code = TYPES[ty]
    st = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T, row = int(st[-1]), heads * q.width
    xd, xv = rows_on_device(rng.standard_normal((T, row)), row, tt)
    y = H.alloc_matrix(T, row, tt)
    B.tman_attend_i8(xd, row, y, row, code, heads, q.cache, *q.geometry(), q.table_d, q.table.shape[1], up(np.array(lens, dtype=np.int32)), up(st), len(lens), T, 0.125,
                     window, q.ws)
    assert B.tman_read_status(q.ws) == 0
    ref, Bs, S, N, P = io.attend(xv.reshape(T, heads, -1), q.oracle, q.table, lens, st, 0.125, window)
    n = N[:, None, None]
    # (as for other values, but that log2 of a scale of 2^-140 is off by 2^-22 of 140, 2^-15 of the scale)
    tol = io.HALF_STEP[ty] * np.abs(ref) + (2.0 ** -134 if ty == "bf16" else 2.0 ** -25)
    tol = tol + Bs * (2.0 ** -11 + 2.0 ** -14 + 2 * (q.width + 16) * 2.0 ** -23 * S[..., None] + (n / 16 + 64) * 2.0 ** -23) + n * 127 * 2.0 ** -25 * P[..., None]
    within(f64(y), ref.reshape(T, -1), tol.reshape(T, -1))


@pytest.mark.parametrize("exponent", [-60, -104, -113, -118, -124, -128, 60, 110])
@pytest.mark.parametrize("lens,new", [([300], [300]), ([500, 20], [90, 20]), ([300, 40], [3, 1]), ([5000], [2])])
def test_values_of_any_size_of_bf16(lens, new, exponent):
    rng = np.random.default_rng(exponent + 200)
    q = Sequences(io, lens, 16, 1, 64, rng)
    q.append(lens, lens, "bf16", rng, v=rng.standard_normal((sum(lens), 64)) * 2.0 ** exponent)
    check_small(q, lens, new, 2, "bf16", rng)
    check_small(q, lens, new, 2, "bf16", rng, window=70)


@pytest.mark.parametrize("ty,size", [("bf16", 2.0 ** -20), ("bf16", 2.0 ** -90), ("bf16", 2.0 ** 50), ("f16", 2.0 ** -11), ("f16", 1.0)])
@pytest.mark.parametrize("new", [2, 400])
def test_pages_of_zeros_in_front_of_all_others(new, ty, size):
    """Zeros count like their neighbours when there are none in front of them."""
    rng = np.random.default_rng(17)
    n = 700
    q = Sequences(io, [n], 16, 1, 64, rng)
    v = rng.standard_normal((n, 64)) * size
    v[:320] = 0
    v[400:450] = 0
    q.append([n], [n], ty, rng, v=v)
    check_small(q, [n], [new], 1, ty, rng)


@pytest.mark.parametrize("new", [2, 400])
@pytest.mark.parametrize("step", [2.0, -2.0])
def test_value_scales_that_grow_or_shrink_along_the_sequence(new, step):
    """By 2^2 a page over 2^80: probabilities times scales are what counts, and the sums of probabilities are those of all tokens."""
    rng = np.random.default_rng(19)
    n = 640
    q = Sequences(io, [n], 16, 1, 64, rng)
    v = rng.standard_normal((n, 64)) * 2.0 ** (step * (np.arange(n) // 16 - 20))[:, None]
    q.append([n], [n], "bf16", rng, v=v)
    check_small(q, [n], [new], 1, "bf16", rng)


@pytest.mark.parametrize("M", [1, 5, 8])
def test_products_and_attention_over_long_contexts_have_one_workspace_in_turn(M):
    """A decode product leaves codes in the workspace, attention parts of heads that several CTAs share: neither is in the other's way."""
    rng = np.random.default_rng(M)
    lens, K, N = [5000] * M, 18944, 512
    q = Sequences(io, lens, 16, 2, 64, rng)
    q.append(lens, lens, "f16", rng)
    size = max(B.tman_workspace_bytes_attend(64), B.tman_workspace_bytes_i8(B.OP_GEMV, M, K, N))
    q.ws = workspace(size)
    x, w, s = up(rng.standard_normal((M, K))).half(), up(rng.integers(-127, 128, (N, K)).astype(np.int8)), torch.ones(N, device="cuda")
    first = None
    for _ in range(3):
        y = H.alloc_matrix(M, N, torch.float16)
        B.tman_mpgemv_i8(w, K, s * 1e-4, x, K, y, N, B.DTYPE_F16, M, K, N, q.ws)
        first = y if first is None else first
        attend(q, lens, [1] * M, 8, "f16", rng)
        assert torch.equal(y.view(torch.int16), first.view(torch.int16))
