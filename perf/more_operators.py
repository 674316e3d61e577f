"""The attention half of a decoder layer in 8 bits as timed cases: products of 8-bit integers with scales per token and channel, norms
and rotation of query and key heads, appending to and reading from a cache held in 8 bits, and attention over that cache.

Formulas.
  tokens    a_scale = max|x| / 127 of a row (1 for a row of zeros), a = round(x / a_scale), to nearest even, division in 32 bits
  product   y[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k]
  heads     z = x / sqrt(mean(x^2) + eps) * weight for each head; then pairs (i, i + rot/2) (or 2i, 2i + 1) of the first `rot` values are
            turned by the angle position * inv_freq[i]
  cache     pages of `page` tokens; a page has one scale for the keys and one for the values of each head.  Tokens appended to a page
            raise its scale to max|new| / 127 where that is more; codes that are there already become round(code * old / new)
  attention softmax(scale * q . k) v for each new token over its sequence up to itself (the last `window` tokens, if not 0); a key or
            value is code * scale of its page

A case is a dict of plain values:
  op      "gemv"    tman_mpgemv_i8: 16-bit rows, quantized in the call, M in 1..8
          "linear"  tman_quantize_tokens_i8, then tman_mpgemm_i8
          "heads"   tman_norm_rotate of T tokens
          "append"  tman_append_i8 of each sequence's last tokens, then tman_read_cache_i8 of the pages that changed
          "attend"  tman_attend_i8 over a filled cache
  M, K, N, pad          of products; a row of x is `pad` values longer than K
  T, heads, kv, D, rot  tokens, query and key heads, their width, how much of it is turned
  S, len, new, page     sequences, the longest one's tokens, how many of them are new at most, tokens a page
  dtype   "f16" or "bf16"
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
MAX_FLOPS = 2.0 * 8192 * 18944 * 3584            # the largest listed product
MAX_CELLS = 18944 * 3584
MAX_CACHE = 32 * 32768 * 4 * 128                  # key values of the largest listed cache, every sequence counted as long as the longest
MAX_SCORES = 2 * 32 * 2048 * 4096
EPS = 1e-6


def listed():
    return [
        # One token through the smallest projection of a layer (key or value): fixed costs of a decode call.
        dict(name="gemv_m1_4096x1024", op="gemv", M=1, K=4096, N=1024, dtype="f16", pad=0),
        # The widest decode batch through the long reduction of a down projection: the weights' bytes.
        dict(name="gemv_m8_14336x4096", op="gemv", M=8, K=14336, N=4096, dtype="bf16", pad=0),
        # A batch just beyond the decode call's rows, or a very short prompt.
        dict(name="linear_m40_4096x14336", op="linear", M=40, K=4096, N=14336, dtype="f16", pad=0),
        # An ordinary prompt of odd length through an attention projection, from rows of a wider matrix.
        dict(name="linear_m777_3584x4608", op="linear", M=777, K=3584, N=4608, dtype="bf16", pad=64),
        # A long batch of prompts through the longest reduction.
        dict(name="linear_m8192_18944x3584", op="linear", M=8192, K=18944, N=3584, dtype="f16", pad=0),
        # One token's query and key heads: the smallest call.
        dict(name="heads_t1_32x8", op="heads", T=1, heads=32, kv=8, D=128, rot=128, adjacent=False, norm=True, dtype="bf16"),
        # A long prompt's, at far positions.
        dict(name="heads_t8191_28x4", op="heads", T=8191, heads=28, kv=4, D=128, rot=128, adjacent=False, norm=True, dtype="f16"),
        # A decode step of 64 sequences: a token each, into pages that are partly full.
        dict(name="append_s64_new1", op="append", S=64, len=4000, new=1, page=16, kv=8, D=128, dtype="bf16"),
        # Two prompts into the cache.
        dict(name="append_s2_new4096", op="append", S=2, len=4100, new=4096, page=64, kv=8, D=128, dtype="f16"),
        # One user's decode step, short context: latency.
        dict(name="attend_s1_len500", op="attend", S=1, len=500, new=1, page=16, heads=32, kv=8, D=128, window=0, dtype="f16"),
        # A decode step of many sequences of very different lengths: the cache's bytes.
        dict(name="attend_s32_len32768", op="attend", S=32, len=32768, new=1, page=16, heads=28, kv=4, D=128, window=0, dtype="bf16"),
        # The second half of two prompts on top of what the cache holds of the first.
        dict(name="attend_s2_new2048", op="attend", S=2, len=4096, new=2048, page=64, heads=32, kv=8, D=128, window=0, dtype="f16"),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    op = rng.choice(("gemv", "gemv", "linear", "linear", "heads", "append", "attend", "attend", "attend"))
    dtype = rng.choice(("f16", "bf16"))
    if op in ("gemv", "linear"):
        K = _log(rng, 256, 18944, 16)
        N = _log(rng, 64, min(32768, MAX_CELLS // K), rng.choice((1, 8, 64)))
        M = rng.randint(1, 8) if op == "gemv" else _log(rng, 1, min(8192, int(MAX_FLOPS / (2.0 * K * N))))
        return dict(op=op, M=M, K=K, N=N, dtype=dtype, pad=rng.choice((0, 0, 8, 264)))
    heads, kv = rng.choice(((32, 8), (28, 4), (16, 16), (16, 2), (20, 1)))
    D = rng.choice((64, 128, 128, 256))
    if op == "heads":
        return dict(op=op, T=_log(rng, 1, 8192 * 32 * 128 // (heads * D)), heads=heads, kv=kv, D=D, rot=rng.choice((D, D, D // 2)),
                    adjacent=rng.random() < 0.3, norm=rng.random() < 0.7, dtype=dtype)
    page = rng.choice((16, 32, 64))
    if op == "append":
        S = _log(rng, 1, 64)
        n = _log(rng, 1, 4096 // S if S > 1 else 8192)
        return dict(op=op, S=S, len=n + rng.randint(0, 200), new=n, page=page, kv=kv, D=D, dtype=dtype)
    S = _log(rng, 1, 64)
    n = rng.choice((1, 1, rng.randint(2, 8), _log(rng, 9, 2048)))
    most = min(MAX_CACHE // (S * kv * D), MAX_SCORES // (S * heads * n), 131072)
    if most < n:
        n = 1
        most = MAX_CACHE // (S * kv * D)
    length = _log(rng, n, most)
    return dict(op=op, S=S, len=length, new=n, page=page, heads=heads, kv=kv, D=D,
                window=rng.choice((0, 0, 0, max(1, length // 3))), dtype=dtype)


def _lengths(c):
    """Tokens and new tokens of each sequence: the first is the longest, the others spread over [0.3, 1] and [0.5, 1] of it."""
    spread = [(i * 0.6180339887498949) % 1.0 for i in range(c["S"])]
    lens = [max(1, int(c["len"] * (1.0 - 0.7 * s))) for s in spread]
    return lens, [min(n, max(1, int(c["new"] * (1.0 - 0.5 * s)))) for n, s in zip(lens, spread)]


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _rows(rows, K, pad, dtype, g):
    """A normal hidden state with 1 % of channels 20 times as large, in a matrix whose rows are `pad` longer."""
    x = torch.randn(rows, K + pad, generator=g, device="cuda")
    x[:, torch.randperm(K, generator=g, device="cuda")[: max(1, K // 100)]] *= 20.0
    return x.to(dtype)


def _keys_values(rows, kv, D, dtype, g):
    """Keys with a few loud channels a head, values with tokens of different sizes."""
    k = torch.randn(rows, kv, D, generator=g, device="cuda")
    k *= 1.0 + 7.0 * (torch.rand(kv, D, generator=g, device="cuda") < 0.03)
    v = torch.randn(rows, kv, D, generator=g, device="cuda") * (0.25 + torch.rand(rows, kv, 1, generator=g, device="cuda"))
    return k.to(dtype), v.to(dtype)


def _table(lens, page, g):
    """Pages of each sequence, scattered over the cache, and how many there are."""
    counts = [(n + page - 1) // page for n in lens]
    perm = torch.randperm(sum(counts), generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(counts)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = perm[at:at + n]
        at += n
    return table, at


def _starts(counts):
    out = torch.zeros(len(counts) + 1, dtype=torch.int32)
    out[1:] = torch.cumsum(torch.tensor(counts), 0)
    return out.cuda()


def _cache(s, lens, kv, D, page, dtype, g):
    """A cache with `lens` tokens of each sequence in it: codes and scales, or the library's buffer, which gets them as a program's
    prompts would."""
    full = torch.tensor(lens, dtype=torch.int32, device="cuda")
    rows = _starts(lens)
    k, v = _keys_values(sum(lens), kv, D, dtype, g)
    if own:
        from paper_2511_11248_b200 import binding as B
        s["cache"] = torch.zeros(B.tman_cache_bytes_i8(s["pages"], page, kv, D), dtype=torch.uint8, device="cuda")
        s["ws"] = torch.empty(B.tman_workspace_bytes_attend(D), dtype=torch.uint8, device="cuda")
        B.tman_workspace_init(s["ws"])
        B.tman_append_i8(s["cache"], s["pages"], page, kv, D, k, kv * D, v, kv * D, _code(dtype), s["table"], s["table"].shape[1],
                         full, rows, len(lens), sum(lens), s["ws"])
    else:
        for name in ("k", "v"):
            s["codes_" + name] = torch.zeros(s["pages"], page, kv, D, dtype=torch.int8, device="cuda")
            s["scale_" + name] = torch.zeros(s["pages"], kv, device="cuda")
        _append(s, k, v, full, rows, sum(lens), page)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, op, dtype = case, case["op"], DTYPES[case["dtype"]]
    s = {"case": c, "dtype": dtype}
    if own:
        from paper_2511_11248_b200 import binding as B
    if op in ("gemv", "linear"):
        M, K, N = c["M"], c["K"], c["N"]
        s["x"] = _rows(M, K, c["pad"], dtype, g)
        s["w"] = torch.randint(-127, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
        s["w_scale"] = (0.5 + torch.rand(N, generator=g, device="cuda")) * 2e-4
        if own:
            s["y"] = torch.empty(M, N, dtype=dtype, device="cuda")
            s["ws"] = torch.empty(B.tman_workspace_bytes_i8(B.OP_GEMV if op == "gemv" else B.OP_GEMM, M, K, N), dtype=torch.uint8, device="cuda")
            B.tman_workspace_init(s["ws"])
            if op == "linear":
                s["a"] = torch.empty(M, K, dtype=torch.int8, device="cuda")
                s["a_scale"] = torch.empty(M, device="cuda")
    elif op == "heads":
        T, D, n = c["T"], c["D"], c["heads"] + c["kv"]
        s["x"] = torch.randn(T, (n + c["kv"]) * D, generator=g, device="cuda").to(dtype)          # q, k and v side by side
        if c["norm"]:
            s["q_weight"], s["k_weight"] = ((0.5 + torch.rand(D, generator=g, device="cuda")).to(dtype) for _ in range(2))
        first = int(torch.randint(0, 120000, (1,), generator=g, device="cuda"))
        s["positions"] = torch.arange(first, first + T, dtype=torch.int32, device="cuda")
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])).float()
        if own:
            s["y"] = torch.empty(T, n * D, dtype=dtype, device="cuda")
    else:
        lens, new = _lengths(c)
        s["table"], s["pages"] = _table(lens, c["page"], g)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["starts"], s["T"] = _starts(new), sum(new)
        kv, D, page = c["kv"], c["D"], c["page"]
        if op == "append":
            old = [a - b for a, b in zip(lens, new)]
            _cache(s, old, kv, D, page, dtype, g)
            s["k"], s["v"] = _keys_values(s["T"], kv, D, dtype, g)
            changed = [a - b // page * page for a, b in zip(lens, old)]          # tokens of the pages that change
            s["read_starts"], s["read_T"] = _starts(changed), sum(changed)
            if own:
                s["out"] = [torch.empty(s["read_T"], kv * D, dtype=dtype, device="cuda") for _ in range(2)]
        else:
            _cache(s, lens, kv, D, page, dtype, g)
            s["q"] = (torch.randn(s["T"], c["heads"] * D, generator=g, device="cuda") * 1.5).to(dtype)
            if own:
                s["y"] = torch.empty(s["T"], c["heads"] * D, dtype=dtype, device="cuda")
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------


def _quantize_tokens(x):
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.where(top > 0, top / 127.0, 1.0)
    return torch.round(x / scale).clamp(-127, 127), scale


def _places(s, lens, starts, T, page):
    """Sequence, position, page and slot of each row: a sequence's rows are its last tokens."""
    counts = starts[1:] - starts[:-1]
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), counts, output_size=T)
    pos = lens[seq] - starts[seq + 1] + torch.arange(T, device="cuda", dtype=torch.int32)
    return seq, pos.long(), s["table"][seq, (pos // page).long()].long(), (pos % page).long()


def _append(s, k, v, lens, starts, T, page):
    seq, pos, at, slot = _places(s, lens, starts, T, page)
    for name, x in (("k", k.float()), ("v", v.float())):
        x = x.view(T, -1, s["codes_" + name].shape[-1])
        codes, scale = s["codes_" + name], s["scale_" + name]
        top = torch.zeros_like(scale).index_reduce_(0, at, x.abs().amax(-1), "amax")
        fresh = torch.zeros(len(scale), dtype=torch.bool, device="cuda")
        fresh[at[slot == 0]] = True
        old = torch.where(fresh[:, None], 0.0, scale)
        touched = torch.zeros_like(fresh)
        touched[at] = True
        both = torch.where(touched[:, None], torch.maximum(old, top / 127.0), scale)
        partly = torch.nonzero(touched & ~fresh)[:, 0]
        ratio = torch.where(both[partly] > 0, old[partly] / both[partly], 0.0)
        codes[partly] = torch.round(codes[partly].float() * ratio[:, None, :, None]).to(torch.int8)
        d = both[at][..., None]
        codes[at, slot] = torch.where(d > 0, torch.round(x / d), 0.0).clamp(-127, 127).to(torch.int8)
        scale.copy_(both)


def _heads(s, c):
    T, D, rot, n = c["T"], c["D"], c["rot"], c["heads"] + c["kv"]
    x = s["x"][:, : n * D].float().view(T, n, D)
    if c["norm"]:
        w = torch.cat((s["q_weight"].float().expand(c["heads"], D), s["k_weight"].float().expand(c["kv"], D)))
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = x.clone()
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if c["adjacent"] else (slice(0, rot // 2), slice(rot // 2, rot))
    out[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    out[..., hi] = x[..., hi] * cos + x[..., lo] * sin
    return out.view(T, n * D)


def _attend(s, c):
    S, T, heads, kv, D, page = c["S"], s["T"], c["heads"], c["kv"], c["D"], c["page"]
    pages = s["table"].clamp(min=0).long()
    L, most = pages.shape[1] * page, c["new"]
    k, v = ((s["codes_" + n][pages].float() * s["scale_" + n][pages][:, :, None, :, None]).view(S, L, kv, D) for n in ("k", "v"))
    seq, pos, _, _ = _places(s, s["lens"], s["starts"], T, page)
    row = torch.arange(T, device="cuda") - s["starts"][seq].long()
    q = torch.zeros(S, most, heads, D, device="cuda")
    q[seq, row] = s["q"].float().view(T, heads, D)
    where = torch.zeros(S, most, dtype=torch.long, device="cuda")
    where[seq, row] = pos
    score = torch.matmul(q.view(S, most, kv, heads // kv, D).permute(0, 2, 3, 1, 4).reshape(S, kv, -1, D), k.permute(0, 2, 3, 1))
    score = score.view(S, kv, heads // kv, most, L) * (1.0 / math.sqrt(D))
    key = torch.arange(L, device="cuda")
    seen = key <= where[..., None]
    if c["window"]:
        seen &= key > where[..., None] - c["window"]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    score.exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(S, kv, -1, L), v.permute(0, 2, 1, 3)).view(S, kv, heads // kv, most, D) / total
    return out.permute(0, 3, 1, 2, 4).reshape(S, most, heads * D)[seq, row]


# ---- one pass ---------------------------------------------------------------------------------------------------------


def _code(dtype):
    from paper_2511_11248_b200 import binding as B
    return B.DTYPE_F16 if dtype == torch.float16 else B.DTYPE_BF16


def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        from paper_2511_11248_b200 import binding as B
        dt = _code(s["dtype"])
        if op in ("gemv", "linear"):
            M, K, N = c["M"], c["K"], c["N"]
            if op == "gemv":
                B.tman_mpgemv_i8(s["w"], K, s["w_scale"], s["x"], K + c["pad"], s["y"], N, dt, M, K, N, s["ws"])
            else:
                B.tman_quantize_tokens_i8(s["x"], K + c["pad"], dt, M, K, s["a"], s["a_scale"])
                B.tman_mpgemm_i8(s["w"], K, s["w_scale"], s["a"], s["a_scale"], s["y"], N, dt, M, K, N, s["ws"])
            return s["y"]
        if op == "heads":
            n = (c["heads"] + c["kv"]) * c["D"]
            B.tman_norm_rotate(s["x"], n + c["kv"] * c["D"], s["y"], n, dt, c["T"], c["heads"], c["kv"], c["D"], c["rot"],
                               int(c["adjacent"]), s.get("q_weight"), s.get("k_weight"), EPS, s["positions"], s["inv_freq"])
            return s["y"]
        kv, D, page, table = c["kv"], c["D"], c["page"], s["table"]
        if op == "append":
            B.tman_append_i8(s["cache"], s["pages"], page, kv, D, s["k"], kv * D, s["v"], kv * D, dt, table, table.shape[1],
                             s["lens"], s["starts"], c["S"], s["T"], s["ws"])
            k, v = s["out"]
            B.tman_read_cache_i8(s["cache"], s["pages"], page, kv, D, table, table.shape[1], s["lens"], s["read_starts"], c["S"],
                                 s["read_T"], k, kv * D, v, kv * D, dt, s["ws"])
            return {"k": k, "v": v}
        B.tman_attend_i8(s["q"], c["heads"] * D, s["y"], c["heads"] * D, dt, c["heads"], s["cache"], s["pages"], page, kv, D, table,
                         table.shape[1], s["lens"], s["starts"], c["S"], s["T"], 1.0 / math.sqrt(D), c["window"], s["ws"])
        return s["y"]
    if op in ("gemv", "linear"):
        a, scale = _quantize_tokens(s["x"][:, : c["K"]].float())
        return (torch.matmul(a, s["w"].float().T) * scale * s["w_scale"]).to(s["dtype"])
    if op == "heads":
        return _heads(s, c).to(s["dtype"])
    if op == "append":
        _append(s, s["k"], s["v"], s["lens"], s["starts"], s["T"], c["page"])
        _, _, at, slot = _places(s, s["lens"], s["read_starts"], s["read_T"], c["page"])
        return {n: (s["codes_" + n][at, slot].float() * s["scale_" + n][at][..., None]).view(s["read_T"], -1).to(s["dtype"]) for n in ("k", "v")}
    return _attend(s, c).to(s["dtype"])


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------


def exact(case, seed):
    c, op = case, case["op"]
    if op in ("gemv", "linear"):
        s = prepare(case, seed)
        x = s["x"].double()[:, : c["K"]]
        unit = x.abs().amax(1)
        unit = torch.where(unit == 0, 1.0, (unit / 127).float().double())
        sums = torch.einsum("mk,nk->mn", torch.round(x / unit[:, None]), s["w"].double())
        return torch.einsum("mn,m,n->mn", sums, unit, s["w_scale"].double())
    if op == "heads":
        s = prepare(case, seed)
        D, rot, out = c["D"], c["rot"], []
        a = torch.outer(s["positions"].double(), s["inv_freq"].double())
        turn = torch.polar(torch.ones_like(a), a)[:, None, :]
        for i, (h, w) in enumerate(((c["heads"], "q_weight"), (c["kv"], "k_weight"))):
            x = s["x"].double()[:, i * c["heads"] * D:][:, : h * D].reshape(-1, h, D)
            if c["norm"]:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * s[w].double()
            pairs = x[..., :rot].reshape(-1, h, rot // 2, 2) if c["adjacent"] else x[..., :rot].reshape(-1, h, 2, rot // 2).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z.flatten(-2) if c["adjacent"] else z.transpose(-1, -2).flatten(-2)
            out.append(torch.cat((z, x[..., rot:]), -1).flatten(1))
        return torch.cat(out, 1)
    # sequence by sequence and page by page; the inputs as the plain form draws them
    page = c["page"]
    lens, new = _lengths(c)
    if op == "append":
        g = torch.Generator(device="cuda").manual_seed(seed)
        _table(lens, page, g)
        old = [a - b for a, b in zip(lens, new)]
        before, after = (_keys_values(sum(n), c["kv"], c["D"], DTYPES[c["dtype"]], g) for n in (old, new))
        out = {"k": [], "v": []}
        for i, name in enumerate(("k", "v")):
            o, n = before[i].double(), after[i].double()
            for a, b in zip(torch.split(o, old), torch.split(n, new)):
                head = a[len(a) // page * page:]                   # what the first page that changes holds already
                units = [(head.abs().amax((0, 2)) / 127).float()] if len(head) else []
                both = torch.cat((head, b))
                for at in range(0, len(both), page):
                    part = both[at:at + page]
                    fresh = part if at or not len(head) else part[len(head):]
                    unit = (fresh.abs().amax((0, 2)) / 127).float()
                    if at == 0 and len(head):
                        unit = torch.maximum(unit, units[0])
                        u = units[0].double()[:, None]
                        part = torch.cat((torch.round(torch.round(head / u) * (units[0] / unit).double()[:, None]), torch.round(fresh / unit.double()[:, None])))
                    else:
                        part = torch.round(part / unit.double()[:, None])
                    out[name].append((part * unit.double()[:, None]).flatten(1))
            out[name] = torch.cat(out[name])
        return out
    s = prepare(case, seed)
    if own:
        return None
    out, at = [], 0
    key = torch.arange(max(lens), device="cuda")
    for i, (n, m) in enumerate(zip(lens, new)):
        pages = s["table"][i, : (n + page - 1) // page].long()
        k, v = ((s["codes_" + x][pages].double() * s["scale_" + x].double()[pages][:, None, :, None]).flatten(0, 1)[:n] for x in ("k", "v"))
        q = s["q"][at:at + m].double().view(m, c["kv"], -1, c["D"])
        p = torch.einsum("mhgd,lhd->hgml", q, k) / math.sqrt(c["D"])
        last = torch.arange(n - m, n, device="cuda")[:, None]
        hidden = key[:n] > last
        if c["window"]:
            hidden |= key[:n] <= last - c["window"]
        p = torch.softmax(p.masked_fill(hidden, -math.inf), -1)
        out.append(torch.einsum("hgml,lhd->mhgd", p, v).flatten(1))
        at += m
    return torch.cat(out)


def work(case):
    """Each operator's inputs read once and its outputs written once; products and scores count two operations a pair."""
    c, op = case, case["op"]
    if op in ("gemv", "linear"):
        M, K, N = c["M"], c["K"], c["N"]
        return {"bytes": N * K + 4 * N + 2 * M * (K + N), "flops": 2.0 * M * K * N}
    if op == "heads":
        n = c["T"] * (c["heads"] + c["kv"]) * c["D"]
        return {"bytes": 4 * n, "flops": 8.0 * n}
    lens, new = _lengths(c)
    width = c["kv"] * c["D"]
    if op == "append":
        rows, changed = sum(new), sum(a - (a - b) // c["page"] * c["page"] for a, b in zip(lens, new))
        return {"bytes": 2 * width * (2 * rows + rows + changed + 2 * changed), "flops": 4.0 * width * (rows + changed)}
    seen = sum(min(n, m - 1 + c["window"]) if c["window"] else n for n, m in zip(lens, new))
    pairs = 0.0
    for n, m in zip(lens, new):
        w = c["window"] or n
        k = min(m, max(0, w - (n - m)))               # new tokens that see less than a whole window: n - m + 1, n - m + 2, ...
        pairs += k * (n - m) + k * (k + 1) / 2.0 + (m - k) * w
    return {"bytes": 2 * width * seen + 4 * sum(new) * c["heads"] * c["D"], "flops": 4.0 * pairs * c["heads"] * c["D"]}
