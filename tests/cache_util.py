"""Steps over a paged cache for the tests: made on the host from a seed, run through the C ABI, held against oracle/cache.py."""
from __future__ import annotations

import numpy as np
import torch

import paper_2411_06360_amd as R
from oracle import cache as oracle

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}  # unit roundoff


def rounder(cache):
    return lambda x: torch.from_numpy(np.ascontiguousarray(x)).float().to(DTYPES[cache]).double().numpy()


def plain(x):
    return None if x is None else x.detach().double().cpu().numpy()


def draft(rng, n):
    """Parents of a drafted tree (-1: hangs on the cache)."""
    return [int(rng.integers(-1, i)) if i else -1 for i in range(n)]


class Step:
    """Tensors of a step on `device`; any of them may be changed before run()."""

    def __init__(self, held, new, *, heads=4, kv_heads=2, dim=64, act="f32", cache="bf16", page=16, tree=True, seed=0, device="cuda", spare=0):
        rng = np.random.default_rng([seed, len(held), dim, page])
        g = torch.Generator().manual_seed(seed * 7919 + dim)
        self.heads, self.kv_heads, self.dim, self.act, self.kind, self.page, self.scale = heads, kv_heads, dim, act, cache, page, dim**-0.5
        need = [-(-h // page) for h in held]
        pages, width = sum(need) + 2, max(need + [1]) + spare
        order = rng.permutation(pages)
        table = np.full((len(held), width), -1, np.int32)
        at = 0
        for r, n in enumerate(need):
            table[r, :n] = order[at:at + n]
            at += n
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.tokens, self.max_new = int(start[-1]), max(list(new) + [1])
        mask = None
        if tree:
            mask = np.zeros(self.tokens, np.uint64)
            parents = [p for n in new for p in draft(rng, n)]
            mask[:] = oracle.masks(parents, start, self.tokens)[0]
            mask = torch.from_numpy(mask.view(np.int64)).to(device)
        width = (heads + 2 * kv_heads) * dim
        rows = torch.randn((self.tokens, width), generator=g).to(DTYPES[act]).to(device)
        self.q, self.k, self.v = rows[:, :heads * dim], rows[:, heads * dim:(heads + kv_heads) * dim], rows[:, (heads + kv_heads) * dim:]
        self.out = torch.full((self.tokens, heads * dim), float("nan"), dtype=DTYPES[act], device=device)
        shape = (pages, kv_heads, page, dim)
        self.cache_k, self.cache_v = (torch.randn(shape, generator=g).to(DTYPES[cache]).to(device) for _ in range(2))
        self.table, self.held, self.start, self.mask = torch.from_numpy(table).to(device), torch.tensor(held, dtype=torch.int32, device=device), torch.from_numpy(start).to(device), mask
        self.workspace = None

    def call(self, stream=None):
        cache = R.make_cache(self.cache_k, self.cache_v)
        step = R.make_step(self.table, self.held, self.start, self.tokens, self.max_new, self.mask)
        if self.workspace is None:
            self.workspace = torch.zeros(R.rsr_tree_attention_workspace(cache, step, self.heads), dtype=torch.uint8, device="cuda")
        R.rsr_tree_attention(cache, step, self.q, self.k, self.v, self.out, self.heads, self.scale, self.workspace,
                             torch.cuda.current_stream().cuda_stream if stream is None else stream)

    def run(self):
        self.call()
        torch.cuda.synchronize()
        return plain(self.out)

    def expected(self):
        mask = None if self.mask is None else self.mask.cpu().numpy().view(np.uint64)
        with np.errstate(invalid="ignore", over="ignore"):
            return oracle.attention(plain(self.q), plain(self.k), plain(self.v), plain(self.cache_k), plain(self.cache_v), self.table.cpu().numpy(),
                                    self.held.cpu().numpy(), self.start.cpu().numpy(), mask, self.heads, self.scale, self.max_new, rounder(self.kind))

    def bound(self, expected):
        """What rounding may do to a value.  A score is off by at most dim + 8 roundings of 2^-24 of scale * sum |q| |k| (its sum,
        its parts and its scale) and the exponential by a few more; a weight off by e moves the result by 2 e of the mean of |v|,
        and sums over n weights by n 2^-24.  With 16-bit activations weights and result are rounded to that type as well."""
        out, spread, steep, n = expected
        u, e = ROUND[self.act], 2.0**-24
        off = steep * (self.dim + 8) * e + 8 * e + n * e
        weights = u if self.act != "f32" else 4 * e
        return spread * (2 * off + 2 * weights) + np.abs(out) * u + 1e-30

    def check(self):
        got, expected = self.run(), self.expected()
        want, far = expected[0], self.bound(expected)
        there = ~np.isnan(want)
        assert np.isfinite(got[there]).all(), "a value was not written, or touched what it does not see"
        assert np.isnan(got[~there]).all(), "a row of no request was written"
        error = np.abs(got - want)[there]
        assert (error <= far[there]).all(), f"off by {float((error / far[there]).max()):.3g} times the bound"
        if there.any() and np.linalg.norm(want[there]):
            # rounding is not biased: over all values the root of the mean square is far below the bound
            rel = np.linalg.norm(error) / np.linalg.norm(want[there])
            assert rel <= (4e-6 if self.act == "f32" else ROUND[self.act]), f"relative error {rel:.3g}"
        return got
