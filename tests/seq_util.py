"""Batches of sequences over a paged cache for the tests of the operators over packed token rows."""
import numpy as np
import torch

from gpu_util import TORCH, rand


class Batch:
    """new[s] new tokens of sequence s, ctx[s] keys in all; pages in random order, `spare` of them not used;
    `behind` rows behind the last sequence; `beyond` more page-table columns than needed."""

    def __init__(self, new, ctx, page, kv_heads, d, dtype, seed, token_major=False, spare=2, behind=2, beyond=1, absent=()):
        rng = np.random.default_rng(seed)
        self.new, self.ctx, self.page, self.dtype = list(new), list(ctx), page, dtype
        need = [-(-max(c, 0) // page) for c in ctx]
        self.pages = sum(need) + spare
        order = rng.permutation(self.pages)
        self.table = np.full((len(ctx), max(need + [0]) + beyond), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        for (s, p, value) in absent:       # pages that are not there
            self.table[s, p] = value
        self.q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.kv_len = np.array(ctx, dtype=np.int32)
        self.tokens = int(self.q_start[-1]) + behind
        shape = (self.pages, page, kv_heads, d) if token_major else (self.pages, kv_heads, page, d)
        self.k, k64 = rand(shape, dtype, seed + 1, -1.5, 1.5)
        self.v, v64 = rand(shape, dtype, seed + 2, -1.5, 1.5)
        if token_major:
            self.k, self.v = self.k.permute(0, 2, 1, 3), self.v.permute(0, 2, 1, 3)
            k64, v64 = k64.transpose(0, 2, 1, 3), v64.transpose(0, 2, 1, 3)
        self.k64, self.v64 = np.ascontiguousarray(k64), np.ascontiguousarray(v64)

    def hide_unused(self, value=float("nan")):
        """`value` wherever no sequence's key lies."""
        used = np.zeros((self.pages, self.page), dtype=bool)
        for s, c in enumerate(self.ctx):
            for j in range(max(c, 0)):
                p = self.table[s, j // self.page]
                if 0 <= p < self.pages:
                    used[p, j % self.page] = True
        hide = torch.from_numpy(~used).cuda()[:, None, :, None].expand(self.k.shape)
        for t in (self.k, self.v):
            t[hide] = value
        for a in (self.k64, self.v64):
            a[np.broadcast_to(~used[:, None, :, None], a.shape)] = np.nan
        return self

    def arrays(self):
        return tuple(torch.from_numpy(a).cuda() for a in (self.q_start, self.kv_len, self.table))


def strided(t, extra):
    """The same rows, `extra` values further apart."""
    m, n = t.shape
    buf = torch.full((m, n + extra), float("nan"), dtype=t.dtype, device=t.device)
    buf[:, :n] = t
    return buf[:, :n]


def sentinel(shape, dtype, fill=-77.0):
    return torch.full(shape, fill, dtype=TORCH[dtype], device="cuda")


def elastic_bitwise(op, outs, orc, bits, plans=(1, 2, 3, 8), blocks=(64, 128, 256)):
    """Every shard plan, order, grid and block gives the bits of the unsharded run."""
    for t in outs:
        t.fill_(-77.0)
    op.run()
    torch.cuda.synchronize()
    ref = [bits(t) for t in outs]
    for n in plans:
        if n > op.T:
            continue
        plan = orc.balanced_split(op.T, n)
        for block in blocks:
            for t in outs:
                t.fill_(-77.0)
            for j in reversed(range(n)):
                b, l = plan[j]
                op.launch(b, l, min(l, 37), block)
            torch.cuda.synchronize()
            assert [bits(t) for t in outs] == ref, (n, block)
    return ref
