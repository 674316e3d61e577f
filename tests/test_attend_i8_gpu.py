"""The 8-bit cache and attention over it on the GPU: the cache bit for bit, attention to the roundings that it makes."""
import numpy as np
import pytest
import torch

from i8_common import TYPES, Sequences, f64, rows_on_device, up, within, workspace
from oracle import i8_oracle as io
from paper_2511_11248_b200 import binding as B, helpers as H

pytestmark = pytest.mark.gpu


def live(q, lens):
    used = {}
    for s, n in enumerate(lens):
        for i in range((n + q.page - 1) // q.page):
            used[int(q.table[s][i])] = min(q.page, n - i * q.page)
    return used


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("page,heads,width,lens", [(16, 1, 64, [1]), (16, 2, 128, [16, 17, 3]), (32, 3, 64, [100, 31, 0, 33]), (64, 8, 128, [65, 200]),
                                                   (128, 2, 256, [300, 1, 127]), (16, 1, 192, [47] * 9)])
def test_append_in_pieces_and_read(page, heads, width, lens, ty):
    """Prompts, then a few tokens, then one at a time, of growing and shrinking size: each state as the oracle's."""
    rng = np.random.default_rng(page + heads + width)
    q = Sequences(io, lens, page, heads, width, rng, capacity=max(lens) + 40)
    q.append(lens, lens, ty, rng, pad=16)
    q.check_bytes(live(q, lens))
    for new in ([7] * len(lens), [1] * len(lens), [int(v) for v in rng.integers(0, 5, len(lens))], [1] * len(lens), [16] * len(lens)):
        if sum(new) == 0:
            new[0] = 1
        lens = [a + b for a, b in zip(lens, new)]
        T = sum(new)
        size = np.exp(1.5 * rng.standard_normal((T, 1)))
        q.append(new, lens, ty, rng, k=rng.standard_normal((T, heads * width)) * size, v=rng.standard_normal((T, heads * width)) * size)
        q.check_bytes(live(q, lens))
    assert B.tman_read_status(q.ws) == 0
    tt, code = TYPES[ty]
    T, row = sum(lens), heads * width
    k, v = H.alloc_matrix(T, row + 8, tt), H.alloc_matrix(T, row, tt)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    B.tman_read_cache_i8(q.cache, *q.geometry(), q.table_d, q.table.shape[1], up(np.array(lens, dtype=np.int32)), up(starts), len(lens), T, k, row + 8, v, row, code, q.ws)
    assert B.tman_read_status(q.ws) == 0
    for s, n in enumerate(lens):
        for got, want in zip((k[:, :row], v), q.oracle.tokens(s, q.table, n)):
            want = torch.from_numpy(want.reshape(n, row).astype(np.float32)).to(tt)       # (a product of 7 and 24 bits, rounded to 32 bits and then once more)
            assert torch.equal(got[starts[s]:starts[s + 1]].cpu(), want)


def test_pages_of_zeros_and_of_what_is_no_number():
    rng = np.random.default_rng(2)
    q = Sequences(io, [4, 4, 4], 16, 2, 64, rng, capacity=40)
    z = np.zeros((12, 128))
    z[5, 70] = np.inf                                     # sequence 1, head 1
    q.append([4, 4, 4], [4, 4, 4], "f16", rng, k=z, v=-z)
    q.check_bytes(live(q, [4, 4, 4]))
    q.append([2, 2, 2], [6, 6, 6], "f16", rng)            # zeros rescaled, NaN stays
    q.check_bytes(live(q, [6, 6, 6]))
    q.append([12, 12, 12], [18, 18, 18], "f16", rng)      # over the page's end
    q.check_bytes(live(q, [18, 18, 18]))
    assert B.tman_read_status(q.ws) == 0
    lens = [3, 3, 3]
    q.append(lens, lens, "f16", rng)                      # the pages begin again
    q.check_bytes(live(q, lens))


def attend(q, lens, new, heads, ty, rng, scale=None, window=0, size=1.0, starts=True, q16=None, stream=None):
    tt, code = TYPES[ty]
    st = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T, row = int(st[-1]) + 2, heads * q.width             # two rows behind the last sequence's
    scale = q.width ** -0.5 if scale is None else scale
    x = rng.standard_normal((T, row)) * size if q16 is None else q16
    xd, xv = rows_on_device(x, row + 8, tt)
    y = H.alloc_matrix(T, row + 16, tt)
    given = up(st) if starts else None
    T_call = T if starts else len(lens)
    B.tman_attend_i8(xd, row + 8, y, row + 16, code, heads, q.cache, *q.geometry(), q.table_d, q.table.shape[1], up(np.array(lens, dtype=np.int32)), given,
                     len(lens), T_call, scale, window, q.ws, **({} if stream is None else {"stream": stream}))
    assert B.tman_read_status(q.ws) == 0
    n = int(st[-1])
    got = f64(y[:n, :row])
    assert bool(torch.isnan(y[n:]).all()) and bool(torch.isnan(y[:, row:]).all())
    ref, Bs, S, N, P = io.attend(xv[:n].reshape(n, heads, -1), q.oracle, q.table, lens, st, float(np.float32(scale)), window)
    check(got, ref, Bs, S, N, P, q.width, ty)
    return got


def check(got, ref, Bs, S, N, P, width, ty):
    """A score is off by 2^-23 for each of its width products and a few operations more, of S; a probability by that in both its exponent and the sum's, by
    2^-20 of the exponential function, and by fp16's half step 2^-11, or 2^-25 of the largest, of 127 codes.  Sums of n / 16 tiles and 64 parts."""
    n = N[:, None, None]
    tol = io.HALF_STEP[ty] * np.abs(ref) + 2.0 ** -25 + Bs * (2.0 ** -11 + 2.0 ** -19 + 2 * (width + 16) * 2.0 ** -23 * S[..., None] + (n / 16 + 64) * 2.0 ** -23)
    tol += n * 127 * 2.0 ** -25 * P[..., None]
    T = len(got)
    within(got, ref.reshape(T, -1), tol.reshape(T, -1))


CASES = [
    # page, kv heads, query heads, width, lens, new
    (16, 1, 1, 64, [1], [1]), (16, 8, 32, 128, [500], [1]), (16, 4, 28, 128, [37, 1, 260, 0, 16, 17], [1] * 6), (32, 2, 16, 64, [1000, 3, 90], [1, 1, 1]),
    (64, 1, 20, 128, [130, 700], [1, 1]), (128, 2, 4, 256, [400, 129], [1, 1]), (16, 3, 3, 192, [55, 64], [1, 1]),
    (16, 8, 32, 128, [300, 41], [4, 4]), (16, 2, 14, 128, [90, 5, 16], [5, 0, 16]), (64, 2, 8, 64, [130, 30], [100, 30]), (32, 4, 16, 128, [257], [257]),
    (16, 1, 16, 256, [70], [33]), (16, 2, 2, 128, [5000], [3]), (16, 2, 32, 128, [129], [129]), (64, 1, 8, 192, [200], [150]),
    (32, 1, 1, 128, [400], [290]), (16, 1, 32, 64, [40, 300, 7, 7], [40, 20, 7, 0]),
]


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("page,kv,heads,width,lens,new", CASES)
def test_attention(page, kv, heads, width, lens, new, ty):
    rng = np.random.default_rng(page + kv + heads + width + sum(lens))
    q = Sequences(io, lens, page, kv, width, rng)
    if sum(lens):
        q.append(lens, lens, ty, rng)
    for window in (0, 1, 20, max(lens)):
        attend(q, lens, new, heads, ty, rng, window=window, size=1.5)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("page,kv,heads,width,lens,new", [
    (16, 1, 4, 128, [1300, 40, 700, 9], [500, 1, 129, 9]), (64, 2, 2, 64, [900, 640], [640, 640]), (128, 1, 2, 192, [700], [300]), (32, 1, 3, 256, [610, 77], [210, 77])])
def test_prompts_beside_single_tokens(page, kv, heads, width, lens, new, ty):
    """Rows of many tiles, over rings of many turns; sequences of one token in the same call."""
    rng = np.random.default_rng(sum(lens) + width)
    q = Sequences(io, lens, page, kv, width, rng)
    q.append(lens, lens, ty, rng)
    for window, size in ((0, 1.5), (0, 12.0), (150, 1.5)):
        attend(q, lens, new, heads, ty, rng, window=window, size=size)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
def test_prompt_over_growing_scores_and_pages_of_zeros(ty):
    """Scores that rise from tile to tile (the running maximum moves every time) and fall again, values of very different sizes, whole pages of zeros."""
    rng = np.random.default_rng(31)
    n = 900
    q = Sequences(io, [n], 16, 1, 64, rng)
    k, v = rng.standard_normal((n, 64)) * 0.1, rng.standard_normal((n, 64))
    k += np.interp(np.arange(n), [0, 600, n], [-4.0, 4.0, -4.0])[:, None] * np.sign(rng.standard_normal(64))
    v[100:300] *= 2.0 ** -9
    v[304:320] = 0
    v[640:656] = 0
    v[700:] *= 20.0
    k[700:] *= 0.5
    q.append([n], [n], ty, rng, k=k, v=v)
    x = np.sign(k[600])[None] * rng.uniform(0.0, 3.0, (402, 1)) + 0.05 * rng.standard_normal((402, 64))
    attend(q, [n], [400], 1, ty, rng, q16=x)


def test_more_sequences_than_threads_and_no_starts():
    rng = np.random.default_rng(8)
    lens = [int(v) for v in rng.integers(0, 60, 900)]
    q = Sequences(io, lens, 16, 1, 64, rng)
    q.append(lens, lens, "f16", rng)
    attend(q, lens, [1] * 900, 4, "f16", rng)
    tt, code = TYPES["f16"]
    xd, xv = rows_on_device(rng.standard_normal((900, 256)), 256, tt)
    y = H.alloc_matrix(900, 256, tt)
    B.tman_attend_i8(xd, 256, y, 256, code, 4, q.cache, *q.geometry(), q.table_d, q.table.shape[1], up(np.array(lens, dtype=np.int32)), None, 900, 900, 0.125, 0, q.ws)
    ref = io.attend(xv.reshape(900, 4, 64), q.oracle, q.table, lens, np.arange(901), 0.125, 0)
    check(f64(y), *ref, 64, "f16")


@pytest.mark.parametrize("ty", ["f16", "bf16"])
def test_long_contexts_are_split_and_joined(ty):
    rng = np.random.default_rng(4)
    lens = [20011, 9000, 130]
    q = Sequences(io, lens, 16, 2, 128, rng)
    q.append(lens, lens, ty, rng)
    got = attend(q, lens, [2, 1, 1], 8, ty, np.random.default_rng(1))
    again = attend(q, lens, [2, 1, 1], 8, ty, np.random.default_rng(1))
    assert np.array_equal(got, again)                     # the workspace is left as it was, and the order of the sums is fixed


@pytest.mark.parametrize("ty", ["f16", "bf16"])
def test_values_of_very_different_sizes(ty):
    """The attended token's page has values 2^-15 of its neighbours'; pages of zeros, large scores; queries of tiny and of huge size."""
    rng = np.random.default_rng(6)
    lens = [96]
    q = Sequences(io, lens, 16, 1, 64, rng)
    k, v = rng.standard_normal((96, 64)), rng.standard_normal((96, 64))
    v[:16] *= 2.0 ** -13
    v[32:48] = 0
    v[64:80] *= 100
    k[5] = 8.0
    k[64:80] *= 0.01
    q.append(lens, lens, ty, rng, k=k, v=v)
    x = np.tile(rng.standard_normal((1, 64)), (3, 2))
    x[0] = 4.0                                            # nearly all on token 5
    for size in (1.0, 2.0 ** -10, 100.0):
        attend(q, lens, [1], 2, ty, rng, q16=x * size)
    if ty == "bf16":
        attend(q, lens, [1], 2, ty, rng, q16=x * 2.0 ** 100, scale=2.0 ** -103)
        attend(q, lens, [1], 2, ty, rng, q16=x * 2.0 ** -110, scale=2.0 ** 107)


def test_what_is_no_number_stays_where_it_is_seen():
    rng = np.random.default_rng(7)
    lens = [40, 40]
    q = Sequences(io, lens, 16, 2, 64, rng)
    k, v = rng.standard_normal((80, 128)), rng.standard_normal((80, 128))
    k[35, 3] = np.nan                                     # sequence 0, head 0, page 2
    v[40 + 2, 70] = np.inf                                # sequence 1, head 1, page 0
    q.append(lens, lens, "f16", rng, k=k, v=v)
    new = [12, 12]
    xd, xv = rows_on_device(rng.standard_normal((24, 256)), 256, torch.float16)
    xd[20, 0] = float("nan")
    y = H.alloc_matrix(24, 256, torch.float16)
    for window in (0, 6):
        y.fill_(7.0)
        B.tman_attend_i8(xd, 256, y, 256, B.DTYPE_F16, 4, q.cache, *q.geometry(), q.table_d, q.table.shape[1], up(np.array(lens, dtype=np.int32)),
                         up(np.array([0, 12, 24], dtype=np.int32)), 2, 24, 0.125, window, q.ws)
        nan = np.isnan(f64(y)).reshape(24, 4, 64)
        want = np.zeros((24, 4, 64), dtype=bool)
        for i in range(12):
            if 28 + i >= 32:
                want[i, :2] = True                        # sees page 2
            if not window:
                want[12 + i, 2:] = True
        want[20, 0] = True
        assert np.array_equal(nan, want)


def test_bad_pages_rows_and_lengths_are_reported_and_touch_nothing():
    rng = np.random.default_rng(11)
    lens = [40, 20, 33]
    q = Sequences(io, lens, 16, 1, 64, rng)
    q.append(lens, lens, "f16", rng)
    whole = q.cache.clone()
    row = torch.randn(3, 64, dtype=torch.float16, device="cuda")
    good = np.array(lens, dtype=np.int32)
    starts = np.array([0, 1, 2, 3], dtype=np.int32)

    def calls(table, lens, starts, T=3):
        out = []
        table, lens, starts = up(table), up(np.array(lens, dtype=np.int32)), up(np.array(starts, dtype=np.int32))
        y = H.alloc_matrix(3, 64, torch.float16, fill=3.0)
        z = H.alloc_matrix(3, 64, torch.float16, fill=3.0)
        B.tman_attend_i8(row, 64, y, 64, B.DTYPE_F16, 1, q.cache, *q.geometry(), table, table.shape[1], lens, starts, 3, T, 0.125, 0, q.ws)
        out.append(B.tman_read_status(q.ws))
        B.tman_workspace_init(q.ws)
        B.tman_read_cache_i8(q.cache, *q.geometry(), table, table.shape[1], lens, starts, 3, T, z, 64, z, 64, B.DTYPE_F16, q.ws)
        out.append(B.tman_read_status(q.ws))
        B.tman_workspace_init(q.ws)
        B.tman_append_i8(q.cache, *q.geometry(), row, 64, row, 64, B.DTYPE_F16, table, table.shape[1], lens, starts, 3, T, q.ws)
        out.append(B.tman_read_status(q.ws))
        B.tman_workspace_init(q.ws)
        q.cache.copy_(whole)
        return out, y, z

    for bad in (-1, q.pages, 2 ** 31 - 1, -2 ** 31):
        t = q.table.copy()
        t[0, 2] = bad                                     # the page of sequence 0's last token
        status, y, z = calls(t, good, starts)
        assert status == [9, 9, 9]
        assert bool((z[0] == 3.0).all()) and not bool((z[1:] == 3.0).any()) and bool(torch.isfinite(y).all())
    for lens_, starts_, T in ([[-1, 20, 33], starts, 3], [[16 * q.table.shape[1] + 1, 20, 33], starts, 3], [good, [-1, 1, 2, 3], 3], [good, [2, 1, 2, 3], 3],
                              [good, [4, 1, 2, 3], 3]):
        status, y, z = calls(q.table, lens_, starts_, T)
        assert status == [9, 9, 9]
        assert not bool((y[2] == 3.0).all()) and bool((z[0] == 3.0).all()) or starts_[0] != 0
    status, y, z = calls(q.table, good, [0, 1, 2, 4])     # the last sequence's rows end behind T
    assert status == [9, 9, 9] and bool((y[2] == 3.0).all()) and bool((z[2] == 3.0).all())
    assert calls(q.table, good, starts)[0] == [0, 0, 0]


def test_more_rows_than_tokens():
    rng = np.random.default_rng(12)
    q = Sequences(io, [3, 20], 16, 1, 64, rng)
    q.append([3, 20], [3, 20], "f16", rng)
    attend(q, [3, 20], [5, 2], 2, "f16", rng)             # rows in front of the first token see nothing: zeros
    x = torch.randn(7, 64, dtype=torch.float16, device="cuda")
    B.tman_append_i8(q.cache, *q.geometry(), x, 64, x, 64, B.DTYPE_F16, q.table_d, q.table.shape[1], up(np.array([3, 20], dtype=np.int32)),
                     up(np.array([0, 5, 7], dtype=np.int32)), 2, 7, q.ws)
    assert B.tman_read_status(q.ws) == 9


@pytest.mark.parametrize("ty", ["f16", "bf16"])
def test_prompts_of_more_rows_than_tokens_and_heads_of_one_key_head(ty):
    """Tiles of rows that begin in front of the first token; many query heads of one key head; a prompt whose last tile of rows has one."""
    rng = np.random.default_rng(14)
    lens, new = [20, 0, 70, 129], [100, 70, 70, 129]
    q = Sequences(io, lens, 16, 1, 64, rng)
    q.append(lens, lens, ty, rng)
    for window in (0, 5):
        attend(q, lens, new, 1, ty, rng, window=window)
    attend(q, lens, [3, 0, 2, 1], 80, ty, rng)
    q128 = Sequences(io, [40], 16, 1, 128, rng)
    q128.append([40], [40], ty, rng)
    attend(q128, [40], [3], 86, ty, rng)                  # 258 rows: two blocks, the second of two rows


def test_two_graphs_with_workspaces_of_their_own_side_by_side():
    """Two captured steps on two streams, replayed at the same time: each with its workspace, over one cache."""
    rng = np.random.default_rng(15)
    lens = [3000, 700]
    q = Sequences(io, lens, 16, 2, 128, rng)
    q.append(lens, lens, "f16", rng)
    st = np.array([0, 1, 2], dtype=np.int32)
    lens_d, starts = up(np.array(lens, dtype=np.int32)), up(st)
    runs = []
    for _ in range(2):
        xd, xv = rows_on_device(rng.standard_normal((2, 1024)), 1024, torch.float16)
        y, ws, stream = H.alloc_matrix(2, 1024, torch.float16), workspace(B.tman_workspace_bytes_attend(128)), torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(3):
                B.tman_attend_i8(xd, 1024, y, 1024, B.DTYPE_F16, 8, q.cache, *q.geometry(), q.table_d, q.table.shape[1], lens_d, starts, 2, 2, 0.09, 0, ws, stream=stream)
        runs.append((graph, stream, xv, y, ws, xd))
    for _ in range(5):
        for graph, stream, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, xv, y, ws, _ in runs:
        assert B.tman_read_status(ws) == 0
        check(f64(y), *io.attend(xv.reshape(2, 8, 128), q.oracle, q.table, lens, st, float(np.float32(0.09)), 0), 128, "f16")


def test_cache_offsets_beyond_32_bits():
    rng = np.random.default_rng(13)
    pages, page, heads, width = 140000, 16, 8, 128        # 4.6 GB
    cache = torch.zeros(B.tman_cache_bytes_i8(pages, page, heads, width), dtype=torch.uint8, device="cuda")
    lens, table = [20, 33], np.array([[139999, 5, -1], [70000, 139998, 3]], dtype=np.int32)
    oracle = io.Cache(6, page, heads, width)
    small = np.array([[0, 1, -1], [2, 3, 4]])
    T, row = 53, heads * width
    starts = np.array([0, 20, 53], dtype=np.int32)
    kd, kv = rows_on_device(rng.standard_normal((T, row)), row, torch.float16)
    vd, vv = rows_on_device(rng.standard_normal((T, row)), row, torch.float16)
    oracle.append(kv.reshape(T, heads, width), vv.reshape(T, heads, width), small, lens, starts)
    ws = workspace(B.tman_workspace_bytes_attend(width))
    args = (pages, page, heads, width)
    seqs = (up(table), 3, up(np.array(lens, dtype=np.int32)))
    B.tman_append_i8(cache, *args, kd, row, vd, row, B.DTYPE_F16, *seqs, up(starts), 2, T, ws)
    k, v = H.alloc_matrix(T, row, torch.float16), H.alloc_matrix(T, row, torch.float16)
    B.tman_read_cache_i8(cache, *args, *seqs, up(starts), 2, T, k, row, v, row, B.DTYPE_F16, ws)
    for s in range(2):
        for got, want in zip((k, v), oracle.tokens(s, small, lens[s])):
            assert torch.equal(got[starts[s]:starts[s + 1]].cpu(), torch.from_numpy(want.reshape(-1, row).astype(np.float32)).half())
    xd, xv = rows_on_device(rng.standard_normal((2, 2 * row)), 2 * row, torch.float16)
    y = H.alloc_matrix(2, 2 * row, torch.float16)
    B.tman_attend_i8(xd, 2 * row, y, 2 * row, B.DTYPE_F16, 16, cache, *args, *seqs, None, 2, 2, 0.0883883, 0, ws)
    assert B.tman_read_status(ws) == 0
    check(f64(y), *io.attend(xv.reshape(2, 16, width), oracle, small, lens, np.arange(3), float(np.float32(0.0883883)), 0), width, "f16")


def test_a_layers_attention_step_captured_and_replayed():
    """Hidden state -> q | k | v product -> norm and rotation -> append -> attention -> output product, on a stream of its own, from one graph: each replay a
    token further, against the oracle run on what the device's own products gave."""
    rng = np.random.default_rng(21)
    S, hidden, heads, kv, width, page = 3, 256, 8, 2, 64, 16
    st = torch.cuda.Stream()
    lens = [15, 3, 40]
    q = Sequences(io, lens, page, kv, width, rng, capacity=80)
    q.append(lens, lens, "f16", rng)
    nq, nk = heads * width, kv * width
    wq, wo = (rng.integers(-127, 128, shape).astype(np.int8) for shape in ((nq + 2 * nk, hidden), (hidden, nq)))
    sq, so = np.full(nq + 2 * nk, 2e-3, dtype=np.float32), np.full(hidden, 2e-3, dtype=np.float32)
    dev = {n: up(v) for n, v in dict(wq=wq, wo=wo, sq=sq, so=so).items()}
    norm = [up(rng.uniform(0.5, 1.5, width)).half() for _ in range(2)]
    freq = (10000.0 ** (-np.arange(0, width, 2) / width)).astype(np.float32)
    freq_d = up(freq)
    x = torch.empty(S, hidden, dtype=torch.float16, device="cuda")
    qkv, out, y = H.alloc_matrix(S, nq + 2 * nk, torch.float16), H.alloc_matrix(S, nq, torch.float16), H.alloc_matrix(S, hidden, torch.float16)
    pre = torch.empty_like(qkv)
    lens_d, pos = up(np.array(lens, dtype=np.int32)), up(np.array(lens, dtype=np.int32) - 1)
    ws = [workspace(B.tman_workspace_bytes_i8(B.OP_GEMV, S, k, n)) for k, n in ((hidden, nq + 2 * nk), (nq, hidden))]
    st.wait_stream(torch.cuda.current_stream())

    def step():
        ld = nq + 2 * nk
        lens_d.add_(1)
        pos.add_(1)
        B.tman_mpgemv_i8(dev["wq"], hidden, dev["sq"], x, hidden, qkv, ld, B.DTYPE_F16, S, hidden, ld, ws[0], stream=st)
        pre.copy_(qkv)
        B.tman_norm_rotate(qkv, ld, qkv, ld, B.DTYPE_F16, S, heads, kv, width, width, 0, *norm, 1e-6, pos, freq_d, stream=st)
        B.tman_append_i8(q.cache, *q.geometry(), qkv[:, nq:], ld, qkv[:, nq + nk:], ld, B.DTYPE_F16, q.table_d, q.table.shape[1], lens_d, None, S, S, q.ws, stream=st)
        B.tman_attend_i8(qkv, ld, out, nq, B.DTYPE_F16, heads, q.cache, *q.geometry(), q.table_d, q.table.shape[1], lens_d, None, S, S, 0.125, 0, q.ws, stream=st)
        B.tman_mpgemv_i8(dev["wo"], nq, dev["so"], out, nq, y, hidden, B.DTYPE_F16, S, nq, hidden, ws[1], stream=st)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step()
    for i in range(20):
        with torch.cuda.stream(st):
            x.copy_(up(rng.standard_normal((S, hidden))).half())
            graph.replay()
        st.synchronize()
        lens = [n + 1 for n in lens]
        ref = io.product(*io.quantize_tokens(f64(x)), wq, sq)
        within(f64(pre), ref, (2.0 ** -11 + 2.0 ** -22) * np.abs(ref) + 2.0 ** -25)
        p = np.array(lens) - 1
        for at, n, w in ((0, heads, norm[0]), (nq, kv, norm[1])):
            r, size = io.norm_rotate(f64(pre)[:, at:at + n * width].reshape(S, n, width), f64(w), 1e-6, p, freq, width, 0)
            within(f64(qkv)[:, at:at + n * width], r.reshape(S, -1), (2.0 ** -11 * np.abs(r) + 2.0 ** -16 * size + 2.0 ** -25).reshape(S, -1))
        held = f64(qkv)
        q.oracle.append(held[:, nq:nq + nk].reshape(S, kv, width), held[:, nq + nk:].reshape(S, kv, width), q.table, lens, np.arange(S + 1))
        check(f64(out), *io.attend(held[:, :nq].reshape(S, heads, width), q.oracle, q.table, lens, np.arange(S + 1), 0.125, 0), width, "f16")
        ref = io.product(*io.quantize_tokens(f64(out)), wo, so)
        within(f64(y), ref, (2.0 ** -11 + 2.0 ** -22) * np.abs(ref) + 2.0 ** -25)
    q.check_bytes(live(q, lens))
    assert B.tman_read_status(q.ws) == 0
