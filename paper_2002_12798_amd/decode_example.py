"""One attention layer of a decoder served from a paged key-value cache: a step takes the new tokens of all requests (whole prompts, then
one token each), and every operator between its two products works on the cache:

    cache_assign   pages, slots and positions of the step's tokens, from the requests' lengths, on the GPU
    gemm_fused     queries, keys and values of the tokens
    cache_append   keys and values into the cache, keys and queries turned to their positions on the way
    cache_attend   each request's newest token over its cache
    gemm_fused     the output projection, which reads the heads [requests, heads, dim] as rows

No length is known on the host.  `python -m paper_2002_12798_amd.decode_example` runs a few steps and compares them with plain attention."""
from __future__ import annotations

import torch

from . import binding as B
from . import device


class PagedAttention:
    def __init__(self, width, heads, kv_heads, dim, requests, longest, page_size=16, theta=10000.0, dtype=torch.bfloat16, seed=0):
        g = torch.Generator().manual_seed(seed)
        dev = device.require_gpu()
        self.heads, self.kv_heads, self.dim, self.width = heads, kv_heads, dim, width
        self.w_qkv = (torch.randn((width, (heads + 2 * kv_heads) * dim), generator=g) * width ** -0.5).bfloat16().to(dev)
        self.w_out = (torch.randn((heads * dim, width), generator=g) * (heads * dim) ** -0.5).bfloat16().to(dev)
        self.rope = device.Rope(theta ** -(torch.arange(dim // 2, device=dev, dtype=torch.float32) / (dim // 2)))
        per_request = -(-longest // page_size)
        pages = requests * per_request
        k, v = (torch.empty((pages, page_size, kv_heads, dim), dtype=torch.bfloat16, device=dev).to(dtype) for _ in range(2))
        self.cache = device.PagedCache(k, v)
        self.table = torch.full((requests, per_request), -1, dtype=torch.int32, device=dev)
        self.length = torch.zeros(requests, dtype=torch.int32, device=dev)
        self.free = torch.randperm(pages, generator=g).int().to(dev)

    def _product(self, x, chain, w):
        m = B.amap_compose([tuple(x.shape)], 2, chain)
        return device.gemm_fused(x.contiguous().view(torch.int16), m, w.view(torch.int16)).view(torch.bfloat16)

    def step(self, x, fresh):
        """x [tokens, width]: the new tokens of request 0, of request 1, ... (fresh[r] of each).  -> each request's output at its newest token,
        0 for a request that has no new one."""
        n, h, k = x.size(0), self.heads, self.kv_heads
        a = device.cache_assign(self.cache.page_size, self.length, fresh, self.table, self.free, n)
        qkv = self._product(x, [], self.w_qkv).view(n, h + 2 * k, self.dim)
        q = device.cache_append(self.cache, qkv[:, h:h + k], qkv[:, h + k:], a.slot, self.rope, a.position, qkv[:, :h])
        newest = (a.begin[1:] - 1).long().clamp(min=0)
        out, _ = device.cache_attend(self.cache, q[newest], self.table, a.length * (fresh > 0))   # (without a new token that row is another request's query)
        self.length = a.length
        self.free = self.free[(torch.arange(self.free.numel(), device=x.device) + a.taken) % self.free.numel()]   # the pages behind those taken come first
        return self._product(out, [("reshape", (out.size(0), h * self.dim))], self.w_out)

    def plain(self, xs):
        """The same for one request's tokens [tokens, width] at its newest one, in 32 bits, without a cache (products rounded as the layer rounds them)."""
        n, h, k, d = xs.size(0), self.heads, self.kv_heads, self.dim
        q, key, v = (xs.float() @ self.w_qkv.float()).bfloat16().float().view(n, h + 2 * k, d).split((h, k, k), 1)
        angle = torch.arange(n, device=xs.device).double()[:, None] * self.rope.freq.double()
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

        def turn(x):
            a, b = x.chunk(2, -1)
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).bfloat16().float()

        q, key = turn(q)[-1], turn(key)
        score = torch.einsum("kgd,nkd->kgn", q.view(k, h // k, d), key) * d ** -0.5
        out = torch.einsum("kgn,nkd->kgd", score.softmax(-1), v).reshape(1, h * d).bfloat16().float()
        return (out @ self.w_out.float())[0]


def run(requests=6, steps=5, width=512, heads=8, kv_heads=2, dim=64, longest=200, seed=3):
    """Prompts of several lengths, then steps of one token for each request: the largest difference from plain attention, by the outputs' size."""
    g = torch.Generator().manual_seed(seed)
    layer = PagedAttention(width, heads, kv_heads, dim, requests, longest + steps)
    history = [torch.empty((0, width), device="cuda") for _ in range(requests)]
    far = 0.0
    for s in range(steps + 1):
        fresh = torch.randint(1, longest + 1, (requests,), generator=g) if s == 0 else torch.ones(requests, dtype=torch.int64)
        x = torch.randn((int(fresh.sum()), width), generator=g).bfloat16().cuda()
        y = layer.step(x, fresh.int().cuda())
        for r, part in enumerate(x.split(fresh.tolist())):
            history[r] = torch.cat([history[r], part.float()])
            want = layer.plain(history[r])
            far = max(far, ((y[r].float() - want).abs().max() / want.abs().max()).item())
    return far


if __name__ == "__main__":
    print(f"largest difference from plain attention: {run():.2g} of the largest output")
