"""Attention over a paged cache by its definition, in 64 bits on the CPU: the oracle of the paged tests, and the random caches they use."""
import math

import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}        # the largest relative error of one rounding


def pages_of(tokens, page):
    return -(-tokens // page)


class World:
    """A cache and a batch of requests [(past, new), ...] on the CPU; `device()` is the library's side of it."""

    def __init__(self, requests, dtype="bf16", dim=128, page=16, kv_heads=2, group=4, layout="thd", spare=3, seed=0, fused=False,
                 wide=2, stale=float("nan"), drift=0.0):
        g = torch.Generator().manual_seed(seed)
        self.requests, self.dtype, self.dim, self.page, self.kv_heads, self.group = requests, dtype, dim, page, kv_heads, group
        self.layout, self.fused = layout, fused
        dt = DTYPES[dtype]
        need = [pages_of(p + n, page) for p, n in requests]
        self.pages = sum(need) + spare
        perm = torch.randperm(self.pages, generator=g).to(torch.int32)
        self.table = torch.full((len(requests), max(need, default=0) + wide), -1, dtype=torch.int32)
        at = 0
        for r, k in enumerate(need):
            self.table[r, :k] = perm[at:at + k]
            at += k
        shape = (self.pages, page, kv_heads, dim)
        self.k, self.v = (torch.randn(shape, generator=g).to(dt) for _ in range(2))
        if drift:
            self.k += (drift * torch.randn((self.pages, 1, kv_heads, dim), generator=g)).to(dt)
        # what no request's tokens lie in holds anything
        real = torch.zeros((self.pages, page), dtype=torch.bool)
        for r, (p, n) in enumerate(requests):
            for j in range(need[r]):
                real[self.table[r, j].long(), :min(page, p + n - j * page)] = True
        self.k[~real], self.v[~real] = stale, stale
        self.count = real.sum(1)
        self.query_start = torch.tensor([0] + list(np.cumsum([n for _, n in requests], dtype=np.int64)), dtype=torch.int32)
        self.kv_lens = torch.tensor([p + n for p, n in requests], dtype=torch.int32)
        self.tokens = int(self.query_start[-1])
        self.q = torch.randn((self.tokens, kv_heads * group, dim), generator=g).to(dt)
        self.bounds = self.codes = self.code_scale = None

    def make_bounds(self):
        """By the definition, page by page."""
        k = torch.where((torch.arange(self.page) < self.count[:, None])[:, :, None, None], self.k.float(), torch.nan)
        lo, hi = (np.asarray(f(k.numpy(), axis=1)) for f in (np.fmin.reduce, np.fmax.reduce))
        b = np.nan_to_num(np.stack((lo, hi), 2)).astype(np.float32)
        scale = (np.abs(b).max((2, 3)) * np.float32(1.0 / 127.0)).astype(np.float32)
        with np.errstate(all="ignore"):
            codes = np.where(scale[:, :, None, None] > 0, np.rint(b / scale[:, :, None, None]), 0.0)
        self.bounds = torch.from_numpy(b).to(DTYPES[self.dtype])
        self.codes, self.code_scale = torch.from_numpy(codes.astype(np.int8)), torch.from_numpy(scale)

    def cache(self, spd):
        def there(x):
            if self.layout == "thd":
                return x.cuda()
            return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        kept = [None] * 3 if self.bounds is None else [x.cuda() for x in (self.bounds, self.codes, self.code_scale)]
        return spd.PagedCache(there(self.k), there(self.v), *kept)

    def batch(self, spd):
        return spd.PagedBatch(self.query_start.cuda(), self.kv_lens.cuda(), self.table.cuda())

    def queries(self):
        if not self.fused:
            return self.q.cuda()
        wide = torch.full((self.tokens, self.q.shape[1] + 2 * self.kv_heads, self.dim), float("nan"), dtype=self.q.dtype)
        wide[:, :self.q.shape[1]] = self.q
        return wide.cuda()[:, :self.q.shape[1]]

    def place(self, r, t):
        n = int(self.query_start[r + 1] - self.query_start[r])
        kv = min(max(int(self.kv_lens[r]), 0), self.table.shape[1] * self.page)
        return kv - n + t - int(self.query_start[r])

    def attention(self, selected=None, scale=None):
        """(out, lse, room) in 64 bits: room[t, h, d] = sum of weight * |value|, what the rounding of weights is a share of."""
        scale = self.dim ** -0.5 if scale is None else scale
        heads = self.kv_heads * self.group
        out, room = (torch.zeros((self.tokens, heads, self.dim), dtype=torch.float64) for _ in range(2))
        lse = torch.full((self.tokens, heads), -math.inf, dtype=torch.float64)
        for r in range(len(self.requests)):
            for t in range(int(self.query_start[r]), int(self.query_start[r + 1])):
                p = self.place(r, t)
                if p < 0:
                    continue
                where = torch.arange(p + 1)
                number = self.table[r, where // self.page].long()
                there = (number >= 0) & (number < self.pages)
                for j in range(self.kv_heads):
                    keep = there if selected is None else there & torch.isin(where // self.page, selected[t, j].long())
                    if not bool(keep.any()):
                        continue
                    k = self.k[number[keep], where[keep] % self.page, j].double()
                    v = self.v[number[keep], where[keep] % self.page, j].double()
                    h = slice(j * self.group, (j + 1) * self.group)
                    x = (self.q[t, h].double() @ k.T) * scale
                    lse[t, h] = torch.logsumexp(x, -1)
                    w = torch.exp(x - lse[t, h, None])
                    out[t, h], room[t, h] = w @ v, w @ v.abs()
        return out, lse, room

    def selection(self, n_select):
        """The selected pages by the definition: whole numbers, and numpy's stable sort."""
        out = np.full((self.tokens, self.kv_heads, n_select), -1, dtype=np.int32)
        codes, scale = self.codes.numpy().astype(np.int64), self.code_scale.numpy()
        q = self.q.float().numpy().reshape(self.tokens, self.kv_heads, self.group, self.dim)
        for r in range(len(self.requests)):
            for t in range(int(self.query_start[r]), int(self.query_start[r + 1])):
                p = self.place(r, t)
                if p < 0:
                    continue
                visible = p // self.page + 1
                number = self.table[r, :visible].numpy()
                for j in range(self.kv_heads):
                    step = np.abs(q[t, j]).max() * np.float32(1.0 / 127.0)
                    c = np.rint(q[t, j] / step) if step > 0 else np.zeros_like(q[t, j])
                    share = np.float32(1.0) / np.float32(self.group)
                    u = np.rint(np.maximum(c, 0).sum(0).astype(np.float32) * share).astype(np.int64)
                    w = np.rint(np.maximum(-c, 0).sum(0).astype(np.float32) * share).astype(np.int64)
                    there = (number >= 0) & (number < self.pages)
                    at = np.where(there, number, 0)
                    score = (codes[at, j, 1] @ u - codes[at, j, 0] @ w).astype(np.float32) * scale[at, j]
                    score = np.where(there, score, -np.inf)
                    score[0] = score[-1] = np.inf
                    best = np.sort(np.argsort(-score, kind="stable")[:n_select])
                    out[t, j, :best.size] = best
        return torch.from_numpy(out)


def assert_close(world, got, want, what=""):
    """Every weight, and the result, is rounded once to the cache's type: u * room + u * |out|.  Logits are sums of at most 128 products in
    fp32, |logit| below 40 here: 128 * 2^-24 * 40 = 3e-4 at the most, of every weight; sums of up to 10^5 weights in fp32 stay within
    that too.  In f16 a weight below 2^-14 is off by up to 2^-25 of the greatest: 2^-25 * keys * |v| <= 2^-25 * 10^4 * 5."""
    out, lse = (x.double().cpu() for x in got)
    want_out, want_lse, room = want
    u = UNIT[world.dtype]
    empty = torch.isinf(want_lse)
    assert torch.equal(lse[empty], want_lse[empty]), what
    assert bool((out[empty] == 0).all()), what
    off = (out - want_out).abs() / (u * (room + want_out.abs()) + 3e-4 * room + (1.5e-3 if world.dtype == "f16" else 0.0) * u + 1e-30)
    off[empty] = 0
    assert bool(torch.isfinite(out).all()), what
    assert off.numel() == 0 or float(off.max()) <= 1.0, (what, float(off.max()), np.unravel_index(int(off.argmax()), off.shape))
    far = (lse - want_lse).abs()
    far[empty] = 0
    assert far.numel() == 0 or float(far.max()) <= 3e-4, (what, float(far.max()))
