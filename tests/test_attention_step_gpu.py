"""A layer's attention half with nothing between its calls: product, norm and rotation, append, attention, output product, from one graph, the way
a program runs them.  Each kernel may start while the one ahead of it runs; the products are long enough to be running still.  What the steps give is
what the same calls give with a wait for the device behind each, bit for bit, and the heads are the definition's."""
import numpy as np
import pytest
import torch

from i8_common import f64, up, within, workspace
from oracle import i8_oracle as io
from paper_2511_11248_b200 import binding as B, helpers as H

pytestmark = pytest.mark.gpu


class Step:
    """Buffers of one step of S sequences of `new` tokens each; `apart`: the heads go to a matrix of their own."""

    def __init__(self, rng, S, new, hidden, heads, kv, width, apart, before=37, page=16, steps=6):
        self.__dict__.update(S=S, new=new, hidden=hidden, heads=heads, kv=kv, width=width, apart=apart, page=page, T=S * new)
        self.nq, self.nk = heads * width, kv * width
        self.ld, nq, nk, T = self.nq + 2 * self.nk, self.nq, self.nk, self.T
        self.per = (before + new * steps + page - 1) // page
        self.pages = S * self.per
        half = lambda *shape: torch.empty(*shape, dtype=torch.float16, device="cuda")
        self.w = [torch.from_numpy(rng.integers(-127, 128, s).astype(np.int8)).cuda() for s in ((self.ld, hidden), (hidden, nq))]
        self.s = [torch.full((n,), 2e-4, device="cuda") for n in (self.ld, hidden)]
        self.norm = [up(rng.uniform(0.5, 1.5, width)).half() for _ in range(2)]
        self.freq = (10000.0 ** (-np.arange(0, width, 2) / width)).astype(np.float32)
        self.freq_d = up(self.freq)
        self.table = up(rng.permutation(self.pages).astype(np.int32).reshape(S, self.per))
        self.starts = up((np.arange(S + 1) * new).astype(np.int32))
        self.lens = up(np.full(S, before, dtype=np.int32))
        self.pos = up(np.tile(np.arange(before, before + new), S).astype(np.int32) - new)
        self.x, self.qkv, self.turned, self.att, self.y = half(T, hidden), half(T, self.ld), half(T, self.ld), half(T, nq), half(T, hidden)
        self.a, self.a_scale = torch.empty(T, max(hidden, nq), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        self.cache = torch.zeros(B.tman_cache_bytes_i8(self.pages, page, kv, width), dtype=torch.uint8, device="cuda")
        self.wa = workspace(B.tman_workspace_bytes_attend(width))
        op = B.OP_GEMV if T <= 8 else B.OP_GEMM
        self.wp = workspace(max(B.tman_workspace_bytes_i8(op, T, k, n) for k, n in ((hidden, self.ld), (nq, hidden))))
        k, v = (up(rng.standard_normal((S * before, nk))).half() for _ in range(2))
        B.tman_append_i8(self.cache, *self.geometry(), k, nk, v, nk, B.DTYPE_F16, self.table, self.per, self.lens,
                         up((np.arange(S + 1) * before).astype(np.int32)), S, S * before, self.wa)

    def geometry(self):
        return self.pages, self.page, self.kv, self.width

    def product(self, i, x, y, K, N, stream, between):
        if self.T <= 8:
            B.tman_mpgemv_i8(self.w[i], K, self.s[i], x, K, y, N, B.DTYPE_F16, self.T, K, N, self.wp, stream=stream)
        else:
            B.tman_quantize_tokens_i8(x, K, B.DTYPE_F16, self.T, K, self.a, self.a_scale, stream=stream)
            between()
            B.tman_mpgemm_i8(self.w[i], K, self.s[i], self.a, self.a_scale, y, N, B.DTYPE_F16, self.T, K, N, self.wp, stream=stream)
        between()

    def run(self, stream, between=lambda: None):
        self.product(0, self.x, self.qkv, self.hidden, self.ld, stream, between)
        out = self.turned if self.apart else self.qkv
        B.tman_norm_rotate(self.qkv, self.ld, out, self.ld, B.DTYPE_F16, self.T, self.heads, self.kv, self.width, self.width, 0, *self.norm, 1e-6, self.pos, self.freq_d,
                           stream=stream)
        between()
        B.tman_append_i8(self.cache, *self.geometry(), out[:, self.nq:], self.ld, self.qkv[:, self.nq + self.nk:], self.ld, B.DTYPE_F16, self.table, self.per,
                         self.lens, self.starts, self.S, self.T, self.wa, stream=stream)
        between()
        B.tman_attend_i8(out, self.ld, self.att, self.nq, B.DTYPE_F16, self.heads, self.cache, *self.geometry(), self.table, self.per, self.lens, self.starts,
                         self.S, self.T, self.width ** -0.5, 0, self.wa, stream=stream)
        between()
        self.product(1, self.att, self.y, self.nq, self.hidden, stream, between)


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("S,new,hidden,heads,kv,width", [(8, 1, 14336, 32, 8, 128), (1, 1, 14336, 28, 4, 128), (2, 150, 4096, 16, 4, 128), (1, 1500, 4096, 16, 16, 64)])
def test_a_step_without_pauses_is_the_step_with_them(S, new, hidden, heads, kv, width, apart):
    rng = np.random.default_rng(S + new + heads)
    step = Step(rng, S, new, hidden, heads, kv, width, apart)
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        for _ in range(2):                                # (the second time over the first's rows, which its last kernels may read still)
            step.run(st)
    seen = ("qkv", "turned", "att", "y", "cache")
    for _ in range(3):
        x = up(rng.standard_normal((step.T, hidden))).half()
        step.lens.add_(new)
        step.pos.add_(new)
        step.x.copy_(x)
        held, results = step.cache.clone(), []
        for paused in (True, False):
            step.cache.copy_(held)
            for b in (step.qkv, step.turned, step.att, step.y):
                b.fill_(float("nan"))
            torch.cuda.synchronize()
            if paused:
                for _ in range(2):
                    step.run(None, torch.cuda.synchronize)
            else:
                with torch.cuda.stream(st):
                    graph.replay()
                st.synchronize()
            results.append([getattr(step, n).clone() for n in seen])
        for name, a, b in zip(seen, *results):
            assert torch.equal(a.view(torch.int8), b.view(torch.int8)), name
        assert B.tman_read_status(step.wa) == 0 and B.tman_read_status(step.wp) == 0
        # the heads against the definition, from the product alone
        pre = torch.empty_like(step.qkv)
        step.product(0, step.x, pre, hidden, step.ld, None, torch.cuda.synchronize)
        out, pos = f64(step.turned if apart else step.qkv), step.pos.cpu().numpy()
        for at, n, w in ((0, heads, step.norm[0]), (step.nq, kv, step.norm[1])):
            r, size = io.norm_rotate(f64(pre)[:, at:at + n * width].reshape(step.T, n, width), f64(w), 1e-6, pos, step.freq, width, 0)
            within(out[:, at:at + n * width], r.reshape(step.T, -1), (2.0 ** -11 * np.abs(r) + 2.0 ** -16 * size + 2.0 ** -25).reshape(step.T, -1))
