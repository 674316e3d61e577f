"""Shared by the tests of the 8-bit integer operators."""
import numpy as np
import torch

from paper_2511_11248_b200 import binding as B, helpers as H

TYPES = {"f16": (torch.float16, B.DTYPE_F16), "bf16": (torch.bfloat16, B.DTYPE_BF16)}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def up(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def rows_on_device(x, ld, dtype):
    """x [M][K] as the first columns of rows of ld values (NaN behind), and the values that it holds in 64 bits."""
    wide = torch.full((x.shape[0], ld), float("nan"), dtype=dtype, device="cuda")
    wide[:, : x.shape[1]] = up(x).to(dtype)
    return wide, f64(wide[:, : x.shape[1]])


def workspace(nbytes):
    ws = H.guarded_bytes(nbytes, "workspace")
    B.tman_workspace_init(ws)
    return ws


def within(got, ref, tol):
    """|got - ref| <= tol everywhere, NaN and infinities alike."""
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isinf(got), np.isinf(ref))
    fine = np.isfinite(ref)
    assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    worst = np.max(np.abs(got - ref)[fine] / np.broadcast_to(tol, ref.shape)[fine], initial=0.0)
    assert worst <= 1.0, worst


class Sequences:
    """Sequences in a cache on the device and in the oracle: lens tokens, new of them rows of the call, pages scattered."""

    def __init__(self, oracle, lens, page, heads, width, rng, spare=3, capacity=None):
        self.lens, self.page, self.heads, self.width = list(lens), page, heads, width
        counts = [((capacity or n) + page - 1) // page for n in lens]
        self.pages = sum(counts) + spare
        perm = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((len(lens), max(max(counts), 1) + 1), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(counts):
            self.table[s, :n] = perm[at:at + n]
            at += n
        self.oracle = oracle.Cache(self.pages, page, heads, width)
        self.cache = H.guarded_bytes(B.tman_cache_bytes_i8(self.pages, page, heads, width), "cache")
        self.cache.fill_(0x5A)                       # (needs no preparation)
        self.table_d = up(self.table)
        self.ws = workspace(B.tman_workspace_bytes_attend(width))

    def geometry(self):
        return self.pages, self.page, self.heads, self.width

    def append(self, new, lens, dtype, rng, k=None, v=None, pad=0, **kw):
        """`new` random tokens of each sequence, which then has `lens`."""
        tt, code = TYPES[dtype]
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T, row = int(starts[-1]), self.heads * self.width
        k = rng.standard_normal((T, row)) if k is None else k
        v = rng.standard_normal((T, row)) * np.exp(rng.standard_normal((T, 1))) if v is None else v
        kd, kv = rows_on_device(k, row + pad, tt)
        vd, vv = rows_on_device(v, row + pad, tt)
        self.oracle.append(kv.reshape(T, self.heads, -1), vv.reshape(T, self.heads, -1), self.table, lens, starts)
        B.tman_append_i8(self.cache, *self.geometry(), kd, row + pad, vd, row + pad, code, self.table_d, self.table.shape[1], up(np.array(lens, dtype=np.int32)),
                         up(starts), len(lens), T, self.ws, **kw)
        return kd, vd

    def check_bytes(self, used):
        """Codes and scales of the pages in `used` as the oracle has them, slots behind the last token apart."""
        _, page, heads, width = self.geometry()
        codes = self.cache[: self.pages * heads * 2 * page * width].cpu().numpy().view(np.int8)
        want = self.oracle.layout().reshape(self.pages, -1)
        got = codes.reshape(self.pages, -1)
        live = np.zeros(self.oracle.codes.shape, dtype=np.int64)
        for p, n in used.items():
            live[p, :, :, :n] = 1
        keep = self.oracle.codes
        self.oracle.codes = live
        mask = self.oracle.layout().reshape(self.pages, -1) != 0
        self.oracle.codes = keep
        assert np.array_equal(got[mask], want[mask])
        off = B.tman_cache_bytes_i8(*self.geometry()) - self.pages * heads * 8
        scales = self.cache[off: off + self.pages * heads * 8].view(torch.float32).cpu().numpy().reshape(self.pages, heads, 2)
        for p in used:
            assert np.array_equal(scales[p], self.oracle.scales[p], equal_nan=True)
