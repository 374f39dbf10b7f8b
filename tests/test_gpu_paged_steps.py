"""Steps of a serving loop with nothing between them: lengths, tables and counts are updated in place by one call and read
by the next, which may start while the one before it still runs."""
import numpy as np
import pytest
import torch

import paged
from paper_2609_32663_gb300 import dkv
from test_gpu_pages import dev

pytestmark = pytest.mark.gpu


class Loop:
    """Steps over L layers of three sequences, all inputs in hand."""

    def __init__(self, steps, dtype, H=8, Hkv=2, L=2, page=16):
        self.dtype, self.steps, self.L, self.H, self.Hkv = dtype, steps, L, H, Hkv
        ctx = np.random.default_rng(1).integers(0, 200, (L, 3, Hkv))
        new = np.array(steps).sum(0)
        need = int((-(-(ctx + new[None, :, None]) // page) - -(-ctx // page)).sum())
        self.cache = paged.Cache(ctx, page, spare=need, wider=int(new.max()) // page + 2, dtype=dtype, H=H)
        gen = torch.Generator().manual_seed(2)
        self.qkv = [[torch.randn((max(sum(n), 1), H + 2 * Hkv, 128), generator=gen).to(dtype) for _ in range(L)] for n in steps]
        p, c = self.cache.pages, self.cache
        self.start = [dev(c.lens), dev(c.table), dev(c.free), dev([c.count]), c.Kp.cuda(), c.Vp.cuda()]
        self.state = [x.clone() for x in self.start]
        self.dqkv = [[x.cuda() for x in s] for s in self.qkv]
        self.tokens = [dev(n) for n in steps]
        self.cu = dev([0] * 4)
        self.out = [[torch.empty((x.shape[0], H, 128), dtype=dtype, device="cuda") for x in s] for s in self.qkv]
        self.status = dev([0])
        self.pw = torch.empty(dkv.dkv_page_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        self.cw = torch.empty(dkv.dkv_chunk_workspace_bytes(p), dtype=torch.uint8, device="cuda")

    def run(self, status=True):
        ln, table, free, count, Kp, Vp = self.state
        p, H, Hkv, word = self.cache.pages, self.H, self.Hkv, self.status if status else None
        for x, old in zip(self.state, self.start):
            x.copy_(old)
        for i in range(len(self.steps)):
            dkv.dkv_page_tables(p, ln, ln, table, free, count, count, self.pw, tokens=self.tokens[i], cu_tokens=self.cu, status=word)
            for layer in range(self.L):
                d = self.dqkv[i][layer]
                dkv.dkv_chunk_attn(p, layer, d[:, :H], d[:, H:H + Hkv], d[:, H + Hkv:], self.cu, table, ln, Kp, Vp,
                                   self.out[i][layer], self.cw, status=word)

    def expect(self):
        """What every step and layer gives, in 64 bits."""
        c, H, Hkv, want = self.cache, self.H, self.Hkv, []
        for i, n in enumerate(self.steps):
            c.table, c.free, c.count, c.lens = paged.tables_after(c, np.broadcast_to(np.array(n)[None, :, None], (self.L, 3, Hkv)))
            for layer in range(self.L):
                x = self.qkv[i][layer]
                o, size, K, V = paged.attention(c, layer, x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:],
                                                np.concatenate([[0], np.cumsum(n)]), True)
                c.Kp, c.Vp = K.to(self.dtype), V.to(self.dtype)
                want.append((i, layer, sum(n), o, size))
        return want

    def check(self, want):
        torch.cuda.synchronize()
        assert int(self.status) == 0
        for i, layer, T, o, size in want:
            paged.assert_attention(self.out[i][layer][:T], o[:T], size[:T], self.dtype, f"step {i} layer {layer}")
            self.out[i][layer].fill_(float("nan"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_steps_back_to_back(cuda, dtype):
    steps = [[1, 1, 1], [1, 0, 1], [40, 1, 0], [1, 1, 1], [0, 0, 0], [1, 70, 2], [1, 1, 1], [3, 1, 17], [1, 1, 1], [1, 1, 1]]
    loop = Loop(steps, dtype)
    want = loop.expect()
    for _ in range(5):
        loop.run()
    loop.check(want)
    loop.run(status=False)  # without a status word
    loop.check(want)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        loop.run()
    for _ in range(2):
        for _ in range(5):
            graph.replay()
        loop.check(want)
