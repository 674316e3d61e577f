"""Definitions of the 8-bit integer operators in NumPy, in 64 bits where nothing else is said: token quantization, products, norm and rotation of
heads, the paged cache and attention over it.  Shares no code with the CUDA path."""
import numpy as np

HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}       # of a rounding, relative


def quantize_tokens(x):
    """Codes and scales of rows of 16-bit values: quotients in single precision."""
    top = np.abs(x).max(-1)
    with np.errstate(invalid="ignore"):
        scale = np.where(top > 0, np.float32(top) / np.float32(127), np.float32(1)).astype(np.float32)
        scale[~np.isfinite(top)] = np.nan
        q = np.float32(x) / scale[:, None]
    return np.where(np.isnan(scale)[:, None], 0, np.rint(np.nan_to_num(q)).clip(-127, 127)).astype(np.int64), scale


def product(a, a_scale, w, w_scale):
    return (a.astype(np.int64) @ w.astype(np.int64).T) * a_scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)


def norm_rotate(x, weight, eps, positions, inv_freq, rot, adjacent):
    """x [T][heads][width]; weight [width] or None.  Returns the result and the sum of magnitudes that each value is made of."""
    z = x.astype(np.float64)
    if weight is not None:
        z = z / np.sqrt((z * z).mean(-1, keepdims=True) + eps) * weight
    y, size = z.copy(), np.abs(z)
    if rot:
        a = positions.astype(np.float64)[:, None, None] * inv_freq.astype(np.float64)
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if adjacent else (slice(0, rot // 2), slice(rot // 2, rot))
        y[..., lo], y[..., hi] = z[..., lo] * np.cos(a) - z[..., hi] * np.sin(a), z[..., hi] * np.cos(a) + z[..., lo] * np.sin(a)
        size[..., lo] = size[..., hi] = size[..., lo] + size[..., hi]
    return y, size


class Cache:
    """codes [pages][heads][2][page][width], scales [pages][heads][2]."""

    def __init__(self, pages, page, heads, width):
        self.page = page
        self.codes = np.zeros((pages, heads, 2, page, width), dtype=np.int64)
        self.scales = np.zeros((pages, heads, 2), dtype=np.float32)

    def append(self, k, v, table, lens, starts):
        """k, v [T][heads][width]; sequence s gets rows starts[s] .. starts[s + 1] as its last tokens."""
        for s, n in enumerate(lens):
            rows = range(starts[s], starts[s + 1])
            first = n - len(rows)
            for at in sorted({p // self.page for p in range(first, n)}):
                new = [(r, first + i - at * self.page) for i, r in enumerate(rows) if (first + i) // self.page == at]
                here = table[s][at]
                for which, x in enumerate((k, v)):
                    part = np.stack([x[r] for r, _ in new]).astype(np.float32)           # [rows][heads][width]
                    fresh = np.abs(part).max((0, 2)) / np.float32(127)
                    fresh[~np.isfinite(part).all((0, 2))] = np.nan
                    old = self.scales[here, :, which] if new[0][1] > 0 else np.zeros_like(fresh)
                    scale = np.where(np.isnan(old) | np.isnan(fresh), np.float32(np.nan), np.maximum(old, fresh))
                    for h in range(len(scale)):
                        c = self.codes[here, h, which]
                        if new[0][1] > 0 and not scale[h] == old[h]:
                            ratio = old[h] / scale[h] if scale[h] > 0 else np.float32(0)
                            c[: new[0][1]] = np.rint(c[: new[0][1]].astype(np.float32) * ratio)
                        for i, (_, slot) in enumerate(new):
                            c[slot] = np.rint(part[i, h] / scale[h]).clip(-127, 127) if scale[h] > 0 else 0
                        self.scales[here, h, which] = scale[h]

    def tokens(self, s, table, n):
        """Keys and values of a sequence's first n tokens, [n][heads][width] each."""
        pages = [table[s][i] for i in range((n + self.page - 1) // self.page)]
        out = []
        for which in (0, 1):
            parts = [self.codes[p, :, which].transpose(1, 0, 2) * self.scales[p, :, which].astype(np.float64)[:, None] for p in pages]
            out.append(np.concatenate(parts)[:n] if parts else np.zeros((0,) + self.codes.shape[1:2] + self.codes.shape[4:]))
        return out

    def layout(self):
        """Bytes of the codes as the buffer holds them."""
        pages, heads, _, page, width = self.codes.shape
        tok, col = np.meshgrid(np.arange(16), np.arange(width), indexing="ij")
        key = (((col // 64) * 2 + tok // 8) * 32 + (tok % 8) * 4 + (col // 16) % 4) * 16 + col % 16
        val = ((col // 32) * 32 + (col % 8) * 4 + (tok % 8) // 2) * 16 + (col // 8) % 4 * 4 + (tok // 8) * 2 + tok % 2
        tiles = self.codes.reshape(pages, heads, 2, page // 16, 16, width)
        out = np.zeros((pages, heads, 2, page // 16, 16 * width), dtype=np.int8)
        out[:, :, 0][..., key] = tiles[:, :, 0]
        out[:, :, 1][..., val] = tiles[:, :, 1]
        return out.reshape(-1)


def attend(q, cache, table, lens, starts, scale, window):
    """q [T][heads][width] in 64 bits.  Returns y and, for each row and head, what a bound on its rounding errors needs: B = sum p |v| [.., width],
    S = max_j scale sum |q| |k_j|, n = keys seen, P = max_j p_j (scale of j's value page)."""
    T, heads, width = q.shape
    y, B = np.zeros(q.shape), np.zeros(q.shape)
    S, P, N = np.zeros((T, heads)), np.zeros((T, heads)), np.zeros(T)
    for s, n in enumerate(lens):
        k, v = cache.tokens(s, table, n)
        rows = range(starts[s], starts[s + 1])
        group = heads // k.shape[1]
        units = np.array([cache.scales[table[s][j // cache.page], :, 1] for j in range(n)], dtype=np.float64).reshape(n, k.shape[1])
        for i, r in enumerate(rows):
            pos = n - len(rows) + i
            lo, hi = max(0, pos - window + 1) if window else 0, max(pos + 1, 0)
            N[r] = hi - lo
            if hi <= lo:
                continue
            for h in range(heads):
                kh, vh = k[lo:hi, h // group], v[lo:hi, h // group]
                z = scale * (kh @ q[r, h])
                p = np.exp(z - z.max())
                p /= p.sum()
                y[r, h], B[r, h] = p @ vh, p @ np.abs(vh)
                S[r, h] = abs(scale) * (np.abs(kh) @ np.abs(q[r, h])).max()
                P[r, h] = (p * units[lo:hi, h // group]).max()
    return y, B, S, N, P
