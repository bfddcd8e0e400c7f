"""Packed tokens over a paged cache for the tests: seeded data on any device, attention in 64 bits."""
import math

import numpy as np
import torch

from paper_2406_10774_amd import binding as Q

D = 128


class Packed:
    """Sequences of lens[b] cached tokens and new[b] packed ones, pages in random order; slots without a token and packed
    rows behind the last sequence are NaN.  stride: elements between packed rows beyond their heads.  room: tokens that a
    page-table row has room for (kernels are chosen by it)."""

    def __init__(self, lens, new, heads=4, kv_heads=2, S=16, seed=0, stride=0, spare_rows=3, cached=True, device="cuda:0",
                 spread=1.0, room=0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.lens, self.new, self.H, self.Hkv, self.G, self.S = list(lens), list(new), heads, kv_heads, heads // kv_heads, S
        self.B, self.dev = len(lens), device
        pages = [-(-n // S) for n in lens]
        width = max(max(pages) + 2, room // S)
        N = sum(pages) + 3
        ids = rng.permutation(N)
        self.table_np = np.full((self.B, width), ids[-1], np.int32)      # rows' ends: a page that nobody has
        at = 0
        for b in range(self.B):
            self.table_np[b, :pages[b]] = ids[at:at + pages[b]]
            at += pages[b]
        self.cu_np = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.total = int(self.cu_np[-1]) + spare_rows

        def normal(*shape):
            return torch.randn(*shape, device=device, dtype=torch.float32, generator=gen)

        self.k_pool = torch.full((N, kv_heads, S, D), math.nan, device=device, dtype=torch.float16)
        self.v_pool = self.k_pool.clone()
        self.meta = torch.zeros(kv_heads, N, 2, D, device=device, dtype=torch.float16)
        self.table = torch.from_numpy(self.table_np).to(device)
        self.seq_lens = torch.tensor(self.lens, device=device, dtype=torch.int32)
        self.cu = torch.from_numpy(self.cu_np).to(device)
        if cached:
            for b in range(self.B):
                t = torch.arange(self.lens[b], device=device)
                phys = self.table[b].long()[t // S]
                self.k_pool[phys, :, t % S] = (normal(self.lens[b], kv_heads, D) * spread).half()
                self.v_pool[phys, :, t % S] = normal(self.lens[b], kv_heads, D).half()

        def packed(n):
            x = torch.full((self.total, n * D + stride), math.nan, device=device, dtype=torch.float16)
            x[:self.cu_np[-1], :n * D] = normal(int(self.cu_np[-1]), n * D).half()
            return x[:, :n * D].unflatten(1, (n, D))

        self.q, self.k_new, self.v_new = packed(heads), packed(kv_heads), packed(kv_heads)
        self.cache = Q.Cache(self.k_pool, self.v_pool, self.meta, self.table, self.seq_lens, num_heads=heads)

    def results(self, half):
        dtype = torch.float16 if half else torch.float32
        return (torch.full((self.total, self.H, D), 77.0, device=self.dev, dtype=dtype),
                torch.full((self.total, self.H), 77.0, device=self.dev, dtype=torch.float32))

    def workspace(self, total=None):
        n = Q.quest_tokens_workspace_bytes(self.cache, self.total if total is None else total)
        return torch.full((max(n, 16) // 4,), math.nan, device=self.dev, dtype=torch.float32)

    def cached(self, b, h):
        t = torch.arange(self.lens[b], device=self.dev)
        phys = self.table[b].long()[t // self.S]
        return self.k_pool[phys, h, t % self.S].double(), self.v_pool[phys, h, t % self.S].double()

    def rows(self, b):
        return slice(int(self.cu_np[b]), int(self.cu_np[b + 1]))


def attention64(q, k, v, sees, scale):
    """q [n][D] over k, v [m][D] where sees [n][m]: out, lse, sum of |weighted values|, largest sum of |products| and tokens
    of each row.  Values that a row does not see do not count, whatever they are."""
    z = torch.where(sees, q @ k.t() * scale, -math.inf)
    lse = torch.logsumexp(z, -1)
    p = torch.where(sees, (z - torch.where(lse == -math.inf, 0.0, lse)[:, None]).exp(), 0.0)
    size = torch.where(sees, q.abs() @ k.abs().t() * abs(scale), 0.0).amax(-1) if k.shape[0] else torch.zeros_like(lse)
    return p @ v, lse, p @ v.abs(), size, sees.sum(-1)


def check(out, lse, want, half, what, vmax=8.0):
    """The limit: what 128-channel sums, exp2 and sums over n tokens cost in fp32 (eight times the square root of the
    number of 2^-24 roundings); with fp16 outputs half a step, 2^-11, for every weight and again for the output, and
    2^-32 of the largest weight for each of n weights that may fall below fp16's smallest step."""
    o, l, weight, size, n = want
    limit = 8 * (math.sqrt(D) * 2.0 ** -24 * size + 2.0 ** -21 + n.double().sqrt() * 2.0 ** -24)
    bound = limit[:, None] * weight + 1e-30
    if half:
        bound = bound + 2.0 ** -11 * weight + 2.0 ** -11 * o.abs() + n[:, None] * 2.0 ** -32 * vmax + 2.0 ** -25
    off = (out.double() - o).abs()
    assert bool((off <= bound).all()), (what, "out", float((off / bound).max()), float(off.max()))
    empty = l == -math.inf
    assert bool((lse[empty] == -math.inf).all()), (what, "lse of empty rows")
    off = (lse.double() - l)[~empty].abs() / l[~empty].abs().clamp(min=1.0)
    assert bool((off <= limit[~empty]).all()), (what, "lse", float((off / limit[~empty]).max()) if off.numel() else 0)


def check_prompt(p, out, lse, half, scale, what=""):
    for b in range(p.B):
        n, at = p.new[b], p.rows(b)
        if n == 0:
            continue
        position = torch.arange(p.lens[b] - n, p.lens[b], device=p.dev)
        sees = torch.arange(p.lens[b], device=p.dev) <= position[:, None]
        for h in range(p.H):
            k, v = p.cached(b, h // p.G)
            want = attention64(p.q[at, h].double(), k, v, sees, scale)
            check(out[at, h], lse[at, h], want, half, (what, b, h))
    left_alone(p, out, lse)


def left_alone(p, out, lse):
    assert bool((out[p.cu_np[-1]:] == 77).all()) and bool((lse[p.cu_np[-1]:] == 77).all()), "rows behind the last sequence"


def mask_of(sees, words):
    """Boolean [n][n] -> int64 [n][words]."""
    n = sees.shape[0]
    bits = np.zeros((n, words), np.uint64)
    for i in range(n):
        for j in range(n):
            if sees[i, j]:
                bits[i, j // 64] |= np.uint64(1 << (j % 64))
    return bits.view(np.int64)


def random_tree(rng, n, words):
    sees = np.zeros((n, n), bool)
    for i in range(n):
        parent = int(rng.integers(-1, i)) if i else -1
        if parent >= 0:
            sees[i] = sees[parent]
        sees[i, i] = True
    return sees


class Trees:
    """Masks of p's drafted nodes; lists: [B][Hkv][K] pages or None."""

    def __init__(self, p, words=None, seed=0, kind=random_tree, lists=None):
        rng = np.random.default_rng(seed)
        self.words = words or max(1, -(-max(p.new) // 64))
        self.sees = [kind(rng, n, self.words) for n in p.new]
        rows = np.full((p.total, self.words), -1, np.int64)
        for b in range(p.B):
            rows[p.rows(b)] = mask_of(self.sees[b], self.words)
        self.mask = torch.from_numpy(rows).to(p.dev)
        self.lists = None if lists is None else torch.from_numpy(np.ascontiguousarray(lists, np.int32)).to(p.dev)


def check_tree(p, t, out, lse, half, scale, what=""):
    for b in range(p.B):
        n, at = p.new[b], p.rows(b)
        if n == 0:
            continue
        drafted = torch.from_numpy(t.sees[b]).to(p.dev)
        for hk in range(p.Hkv):
            k, v = p.cached(b, hk)
            if t.lists is not None:           # a page listed twice counts twice; entries behind a row's pages are not read
                pages = t.lists[b, hk, :p.table.shape[1]].long()
                pages = pages[(pages >= 0) & (pages < -(-p.lens[b] // p.S))]
                j = (pages[:, None] * p.S + torch.arange(p.S, device=p.dev)).flatten()
                j = j[j < p.lens[b]]
                k, v = k[j], v[j]
            sees = torch.cat([torch.ones(n, k.shape[0], dtype=torch.bool, device=p.dev), drafted], 1)
            k, v = torch.cat([k, p.k_new[at, hk].double()]), torch.cat([v, p.v_new[at, hk].double()])
            for h in range(hk * p.G, (hk + 1) * p.G):
                want = attention64(p.q[at, h].double(), k, v, sees, scale)
                check(out[at, h], lse[at, h], want, half, (what, b, h))
    left_alone(p, out, lse)
