"""The 8-bit integer operators without a GPU: sizes, refusals before any launch, pins of the oracle."""
import ctypes as C

import numpy as np
import pytest

from oracle import i8_oracle as io
from test_f4_abi import Fake, Stream


@pytest.fixture(scope="module")
def lib():
    from paper_2511_11248_b200 import build, binding
    build.build()
    return binding.lib()


def _calls(B, **over):
    """Every call with arguments that are right except for `over`; nothing is launched as long as one is wrong."""
    at = lambda i, size=1 << 24: Fake((1 << 30) + (i << 25), size)
    a = dict(w=at(1), ldw=256, w_scale=at(2), x=at(3), ldx=256, a=at(4), a_scale=at(5), y=at(6), ldy=40, dtype=0, M=4, K=256, N=40, ws=at(7),
             q_heads=2, k_heads=1, width=64, rot=64, weight=at(8), positions=at(9), freq=at(10),
             cache=at(11), pages=10, page=16, kv=2, heads=4, k=at(12), ldk=256, v=at(13), ldv=256, table=at(14), ld_table=3, lens=at(15), starts=at(16), S=2, T=5,
             window=0, q=at(17), ldq=256, out=at(18), ldo=256, stream=Stream())
    a.update(over)
    g = type("A", (), a)
    seqs = (g.table, g.ld_table, g.lens, g.starts, g.S, g.T)
    geo = (g.cache, g.pages, g.page, g.kv, g.width)
    return {
        "tokens": lambda: B.tman_quantize_tokens_i8(g.x, g.ldx, g.dtype, g.M, g.K, g.a, g.a_scale, stream=g.stream),
        "gemv": lambda: B.tman_mpgemv_i8(g.w, g.ldw, g.w_scale, g.x, g.ldx, g.y, g.ldy, g.dtype, g.M, g.K, g.N, g.ws, stream=g.stream),
        "gemm": lambda: B.tman_mpgemm_i8(g.w, g.ldw, g.w_scale, g.a, g.a_scale, g.y, g.ldy, g.dtype, g.M, g.K, g.N, g.ws, stream=g.stream),
        "heads": lambda: B.tman_norm_rotate(g.x, g.ldx, g.out, g.ldo, g.dtype, g.T, g.q_heads, g.k_heads, g.width, g.rot, 0, g.weight, g.weight, 1e-6,
                                            g.positions, g.freq, stream=g.stream),
        "append": lambda: B.tman_append_i8(*geo, g.k, g.ldk, g.v, g.ldv, g.dtype, *seqs, g.ws, stream=g.stream),
        "read": lambda: B.tman_read_cache_i8(*geo, *seqs, g.k, g.ldk, g.v, g.ldv, g.dtype, g.ws, stream=g.stream),
        "attend": lambda: B.tman_attend_i8(g.q, g.ldq, g.out, g.ldo, g.dtype, g.heads, *geo, *seqs, 0.125, g.window, g.ws, stream=g.stream),
    }


PRODUCTS, CACHED, ALL = ("gemv", "gemm"), ("append", "read", "attend"), ("tokens", "gemv", "gemm", "heads", "append", "read", "attend")
odd = lambda i, by: Fake((1 << 30) + (i << 25) + by, 1 << 24)


@pytest.mark.parametrize("over,status,calls", [
    (dict(dtype=2), 3, ALL), (dict(K=0), 2, ("tokens",) + PRODUCTS), (dict(K=248), 2, ("tokens",) + PRODUCTS), (dict(K=131072, ldx=131072, ldw=131072), 2, ("tokens",) + PRODUCTS),
    (dict(M=0), 2, ("tokens",) + PRODUCTS), (dict(M=9), 2, ("gemv",)), (dict(N=0), 2, PRODUCTS), (dict(ldw=240), 2, PRODUCTS), (dict(ldw=264), 2, PRODUCTS),
    (dict(ldx=248), 2, ("tokens", "gemv")), (dict(ldx=260), 2, ("tokens", "gemv", "heads")), (dict(ldy=39), 2, PRODUCTS),
    (dict(w=odd(1, 8)), 2, PRODUCTS), (dict(w_scale=odd(2, 2)), 2, PRODUCTS), (dict(x=odd(3, 8)), 2, ("tokens", "gemv", "heads")), (dict(a=odd(4, 8)), 2, ("tokens", "gemm")),
    (dict(a_scale=odd(5, 2)), 2, ("tokens", "gemm")), (dict(y=odd(6, 1)), 2, PRODUCTS), (dict(ws=odd(7, 16)), 2, PRODUCTS + CACHED), (dict(ws=Fake(1 << 30, 64)), 4, PRODUCTS + CACHED),
    (dict(w=Fake(0, 9)), 1, PRODUCTS), (dict(w_scale=Fake(0, 9)), 1, PRODUCTS), (dict(x=Fake(0, 9)), 1, ("tokens", "gemv", "heads")), (dict(a=Fake(0, 9)), 1, ("tokens", "gemm")),
    (dict(a_scale=Fake(0, 9)), 1, ("tokens", "gemm")), (dict(y=Fake(0, 9)), 1, PRODUCTS), (dict(ws=Fake(0, 9)), 1, PRODUCTS + CACHED),
    (dict(T=0), 2, ("heads",) + CACHED), (dict(width=60), 2, ("heads",)), (dict(width=264, ldx=1024, ldo=1024), 2, ("heads",)), (dict(rot=72), 2, ("heads",)), (dict(rot=80), 2, ("heads",)),
    (dict(q_heads=-1), 2, ("heads",)), (dict(q_heads=0, k_heads=0), 2, ("heads",)), (dict(q_heads=4), 2, ("heads",)), (dict(weight=odd(8, 8)), 2, ("heads",)),
    (dict(positions=Fake(0, 9)), 1, ("heads",)), (dict(freq=Fake(0, 9)), 1, ("heads",)), (dict(out=Fake(0, 9)), 1, ("heads", "attend")), (dict(out=odd(18, 8)), 2, ("heads", "attend")),
    (dict(out=odd(3, 0), ldo=512), 2, ("heads",)),
    (dict(page=8), 3, CACHED), (dict(page=48), 3, CACHED), (dict(width=96), 3, CACHED), (dict(pages=0), 2, CACHED), (dict(kv=0), 2, CACHED), (dict(kv=3), 2, ("attend",)),
    (dict(cache=Fake(1 << 30, 1000)), 4, CACHED), (dict(cache=odd(11, 128)), 2, CACHED), (dict(cache=Fake(0, 1 << 24)), 1, CACHED), (dict(table=Fake(0, 9)), 1, CACHED),
    (dict(lens=Fake(0, 9)), 1, CACHED), (dict(lens=odd(15, 2)), 2, CACHED), (dict(starts=None), 2, CACHED), (dict(S=0), 2, CACHED), (dict(ld_table=0), 2, CACHED),
    (dict(ldk=120), 2, ("append", "read")), (dict(ldv=132), 2, ("append", "read")), (dict(k=odd(12, 2)), 2, ("append", "read")), (dict(v=Fake(0, 9)), 1, ("append", "read")),
    (dict(ldq=248), 2, ("attend",)), (dict(q=odd(17, 2)), 2, ("attend",)), (dict(heads=5), 2, ("attend",)), (dict(heads=0), 2, ("attend",)), (dict(window=-1), 2, ("attend",)),
    (dict(ws=Fake(1 << 30, 1000)), 4, ("attend",)), (dict(T=1 << 30), 2, CACHED), (dict(kv=1, heads=4097, ldq=1 << 20, ldo=1 << 20), 2, ("attend",)),
    (dict(ld_table=1 << 28, S=5), 3, ("attend",))])
def test_wrong_arguments_are_refused_before_any_launch(lib, over, status, calls):
    from paper_2511_11248_b200 import binding as B
    table = _calls(B, **over)
    for name in calls:
        with pytest.raises(B.TmanError) as e:
            table[name]()
        assert e.value.status == status, name


def test_sizes(lib):
    from paper_2511_11248_b200 import binding as B
    assert B.tman_cache_bytes_i8(10, 16, 2, 64) == 10 * 2 * 2 * 16 * 64 + 10 * 2 * 8
    assert B.tman_cache_bytes_i8(200000, 128, 8, 256) == 200000 * 8 * 2 * 128 * 256 + 200000 * 64
    assert B.tman_workspace_bytes_i8(B.OP_GEMV, 8, 4096, 100) >= 256 and B.tman_workspace_bytes_i8(B.OP_GEMM, 9999, 4096, 100) >= 256
    out = C.c_size_t(0)
    assert lib.tman_cache_bytes_i8(1, 16, 1, 64, None) == 1 and lib.tman_workspace_bytes_i8(0, 1, 64, 8, None) == 1 and lib.tman_workspace_bytes_attend(64, None) == 1
    assert lib.tman_workspace_bytes_i8(2, 1, 64, 8, C.byref(out)) == 3 and lib.tman_workspace_bytes_i8(0, 9, 64, 8, C.byref(out)) == 2
    assert lib.tman_workspace_bytes_attend(100, C.byref(out)) == 3 and lib.tman_cache_bytes_i8(1, 16, 65536, 64, C.byref(out)) == 2
    assert B.tman_status_string(9) == "TMAN_ERR_INDEX" and B.STATUS_NAMES[9] == "TMAN_ERR_INDEX"


def test_oracle_of_tokens_and_products():
    x = np.array([[127.0, 0.5, 1.5, -2.5, 0.0], [0.0] * 5, [1.0, np.inf, 0, 0, 0]])
    a, s = io.quantize_tokens(x)
    assert a[0].tolist() == [127, 0, 2, -2, 0] and s[0] == 1 and a[1].tolist() == [0] * 5 and s[1] == 1 and np.isnan(s[2]) and not a[2].any()
    w = np.array([[1, 2, 3, 4, 5]])
    assert io.product(a[:2], s[:2], w, np.array([0.5], dtype=np.float32)).tolist() == [[(127 + 6 - 8) * 0.5], [0.0]]


def test_oracle_of_rotation_keeps_lengths_and_positions_add():
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((1, 1, 16)), np.array([1.0, 0.1, 0.01, 0.001], dtype=np.float32)
    for adjacent in (0, 1):
        y, _ = io.norm_rotate(x, None, 0, np.array([3]), f, 8, adjacent)
        z, _ = io.norm_rotate(y, None, 0, np.array([4]), f, 8, adjacent)
        assert np.allclose(z, io.norm_rotate(x, None, 0, np.array([7]), f, 8, adjacent)[0])
        assert np.allclose((y ** 2).sum(), (x ** 2).sum()) and np.array_equal(y[..., 8:], x[..., 8:])
    n, _ = io.norm_rotate(x, np.full(16, 2.0), 0, np.array([0]), f, 8, 0)
    assert np.allclose((n ** 2).mean(), 4.0)


def test_oracle_of_the_cache():
    c = io.Cache(2, 16, 1, 64)
    k = np.zeros((1, 1, 64))
    k[0, 0, :2] = 127.0, 50.0
    c.append(k, 2 * k, [[1]], [1], [0, 1])
    assert c.scales[1, 0].tolist() == [1.0, 2.0] and c.codes[1, 0, 0, 0, :2].tolist() == [127, 50]
    c.append(2 * k, k, [[1]], [2], [0, 1])                 # the keys' scale doubles: 50 -> 25; the values' stays
    assert c.scales[1, 0].tolist() == [2.0, 2.0] and c.codes[1, 0, 0, :2, :2].tolist() == [[64, 25], [127, 50]]      # (63.5 to even)
    assert c.codes[1, 0, 1, :2, :2].tolist() == [[127, 50], [64, 25]]
    kk, vv = c.tokens(0, [[1]], 2)
    assert kk[1, 0, 0] == 254 and vv[1, 0, 1] == 50
    # every byte of a tile is one token and column's
    c.codes[:] = np.arange(2 * 2 * 16 * 64).reshape(c.codes.shape) % 251 - 125
    for page in range(2):
        for which in range(2):
            at = (page * 2 + which) * 1024
            assert sorted(c.layout()[at:at + 1024]) == sorted(c.codes[page, 0, which].reshape(-1))


def test_oracle_of_attention():
    rng = np.random.default_rng(1)
    c = io.Cache(3, 16, 2, 64)
    c.append(rng.standard_normal((20, 2, 64)), rng.standard_normal((20, 2, 64)), [[2, 0]], [20], [0, 20])
    q = rng.standard_normal((3, 4, 64))
    y, *_ = io.attend(q, c, [[2, 0]], [20], [0, 3], 0.125, 0)
    k, v = c.tokens(0, [[2, 0]], 20)
    p = np.exp(0.125 * k[:19, 1] @ q[1, 3])
    assert np.allclose(y[1, 3], p @ v[:19, 1] / p.sum())
    assert np.allclose(io.attend(q, c, [[2, 0]], [20], [0, 3], 0.125, 1)[0][2, 0], v[19, 0])        # a window of one: the token itself
    assert not io.attend(q, c, [[2, 0]], [0], [0, 3], 0.125, 0)[0].any()
