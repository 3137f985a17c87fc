"""Decoding with drafted trees: a transformer's attention block with ternary weights, several requests at a time.

    python -m examples.tree_decode

A step takes for every request the token that was decided last and a small tree of guesses behind it, through

    rsr_tree_masks      who sees whom, how deep a token hangs (its position)
    rsr_matvec_multi    queries, keys and values of all tokens: one pass over the three index tables
    rsr_head_rotate     norms of their heads, rotated by the positions (with --rotary; else positions have embeddings)
    rsr_tree_attention  over the request's pages and the tree
    rsr_matvec          the block's output, and the scores of the next tokens
    rsr_sample          the tokens chosen by them: the likeliest, or drawn (with --temperature and --top-p)
    rsr_tree_keep       the path that the model itself would have taken
    rsr_cache_slots     room for its tokens
    rsr_cache_append    their keys and values, and no others

so that one step yields as many tokens as guesses were right, plus one, and always those that decoding one by one yields: what a
token is drawn with belongs to its request and position.  Weights are random; the vocabulary is a toy's.
"""
from __future__ import annotations

import argparse
import time
from dataclasses import dataclass
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

import paper_2411_06360_amd as R


@dataclass(frozen=True)
class Config:
    hidden: int = 2560
    heads: int = 20
    kv_heads: int = 5
    vocabulary: int = 512
    k: int = 10
    page_size: int = 64
    pages: int = 256
    pages_per_request: int = 32
    seed: int = 0
    rotary: bool = False  # positions rotate normed heads
    temperature: float = 0.0
    top_p: float = 1.0

    @property
    def head_dim(self) -> int:
        return self.hidden // self.heads


class Weights:
    """Ternary matrices, embeddings of tokens and of positions; on the host, a plain model computes with them too."""

    def __init__(self, c: Config):
        rng = np.random.default_rng(c.seed)
        kv = c.kv_heads * c.head_dim
        shapes = {"q": (c.hidden, c.hidden), "k": (c.hidden, kv), "v": (c.hidden, kv), "o": (c.hidden, c.hidden), "head": (c.hidden, c.vocabulary)}
        self.matrices = {n: rng.integers(-1, 2, s).astype(np.int8) for n, s in shapes.items()}
        self.scale = float(np.sqrt(1.5 / c.hidden))  # of a product: as long as its vector then
        self.tokens = rng.standard_normal((c.vocabulary, c.hidden), dtype=np.float32)
        self.positions = 0.1 * rng.standard_normal((c.page_size * c.pages_per_request, c.hidden), dtype=np.float32)
        self.attention = 2.0  # of what the block adds


class Model:
    """The block on the GPU, with the cache of its requests."""

    def __init__(self, c: Config, w: Weights, requests: int):
        self.c, self.w = c, w
        self.handles = {n: R.rsr_preprocess(m, min(c.k, m.shape[1])) for n, m in w.matrices.items()}
        self.tokens, self.positions = torch.from_numpy(w.tokens).cuda(), torch.from_numpy(w.positions).cuda()
        shape = (c.pages, c.kv_heads, c.page_size, c.head_dim)
        self.keys, self.values = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.cache = R.make_cache(self.keys, self.values)
        ints = {"dtype": torch.int32, "device": "cuda"}
        self.table = torch.full((requests, c.pages_per_request), -1, **ints)
        self.free, self.count, self.left = torch.arange(c.pages, **ints), torch.full((1,), c.pages, **ints), torch.zeros(1, **ints)
        self.held, self.now = torch.zeros(requests, **ints), torch.zeros(requests, **ints)
        self.begin = torch.zeros(requests + 1, **ints)  # where the slots of a request begin
        self.workspace, self.space = (torch.zeros(0, dtype=torch.uint8, device="cuda") for _ in range(2))  # of the attention, and of choosing
        self.rotary = None
        if c.rotary:
            pairs = c.head_dim // 2
            self.rotary = R.make_rotary(1e4 ** -(torch.arange(pairs, dtype=torch.float64) / pairs).cuda(), c.head_dim, eps=1e-6)
        self.uniform = torch.from_numpy(np.random.default_rng(c.seed + 2).random((requests, len(w.positions)), dtype=np.float32)).cuda()

    def close(self) -> None:
        torch.cuda.synchronize()
        for h in self.handles.values():
            R.rsr_destroy(h)
        self.handles = {}

    def product(self, name: str, x):
        out = torch.empty((x.shape[0], self.w.matrices[name].shape[1]), device="cuda")
        R.rsr_matvec(self.handles[name], x, out, x.shape[0], torch.cuda.current_stream().cuda_stream)
        return out.mul_(self.w.scale)

    def guesses(self, width: int) -> List[List[int]]:
        """For every token the likeliest next ones by its embedding alone: what trees are drafted from."""
        return self.product("head", self.tokens).topk(width, dim=1).indices.tolist()

    def forward(self, tokens: Sequence[int], start: Sequence[int], parents: Optional[Sequence[int]] = None):
        """The next token behind each of the requests' new tokens (a chain each, or trees by their parents).  The tokens are not in the
        cache yet: append() brings them there."""
        c, w, stream = self.c, self.w, torch.cuda.current_stream().cuda_stream
        n, kv = len(tokens), c.kv_heads * c.head_dim
        most = max(b - a for a, b in zip(start, start[1:]))
        at = torch.tensor(start, dtype=torch.int32).cuda()
        owner = torch.repeat_interleave(torch.arange(len(start) - 1), torch.tensor(start).diff()).cuda()
        mask, self.start, self.drafted, self.parents = None, at, torch.tensor(tokens, dtype=torch.int32).cuda(), None
        if parents is None:
            depth = torch.arange(n, device="cuda") - at[owner]
        else:
            mask, depth = torch.empty(n, dtype=torch.int64, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
            self.parents = torch.tensor(parents, dtype=torch.int32).cuda()
            R.rsr_tree_masks(self.parents, at, mask, depth, stream)
        position = (self.held[owner] + depth).int()
        x = self.tokens[self.drafted.long()]
        if not c.rotary:
            x = x + self.positions[position.long()]
        q, self.k, self.v = (torch.empty((n, width), device="cuda") for width in (c.hidden, kv, kv))
        R.rsr_matvec_multi([(self.handles["q"], x, q), (self.handles["k"], x, self.k), (self.handles["v"], x, self.v)], n, stream)
        for y in (q, self.k, self.v):
            y.mul_(w.scale)
        if c.rotary:
            R.rsr_head_rotate(self.rotary, q, self.k, position, q, self.k, stream)
        mixed = torch.empty_like(q)
        step = R.make_step(self.table, self.held, at, n, most, mask)
        need = R.rsr_tree_attention_workspace(self.cache, step, c.heads)
        if need > self.workspace.numel():
            self.workspace = torch.zeros(need, dtype=torch.uint8, device="cuda")
        R.rsr_tree_attention(self.cache, step, q, self.k, self.v, mixed, c.heads, c.head_dim ** -0.5, self.workspace, stream)
        scores = self.product("head", x + w.attention * self.product("o", mixed))
        need = R.rsr_sample_workspace(*scores.shape)
        if need > self.space.numel():
            self.space = torch.zeros(need, dtype=torch.uint8, device="cuda")
        self.chosen = torch.empty(n, dtype=torch.int32, device="cuda")
        numbers = {name: torch.full((n,), x, device="cuda") for name, x in (("temperature", c.temperature), ("top_p", c.top_p))}
        R.rsr_sample(scores, self.uniform[owner, position.long()], self.chosen, self.space, stream=stream, **numbers)
        return self.chosen

    def keep(self) -> List[List[int]]:
        """The paths of the last forward()'s trees that agree with what it chose go into the cache; what was found on them."""
        ints = {"dtype": torch.int32, "device": "cuda"}
        rows, found = (torch.empty(self.drafted.numel(), **ints) for _ in range(2))
        add, first = (torch.empty(self.held.numel() + i, **ints) for i in range(2))
        R.rsr_tree_keep(self.drafted, self.chosen, self.parents, self.start, rows, found, add, first, torch.cuda.current_stream().cuda_stream)
        self.append(rows, add)
        tokens, ends = found.tolist(), first.tolist()
        return [tokens[a:b] for a, b in zip(ends, ends[1:])]

    def append(self, rows, add) -> None:
        """Rows of the last forward() go into the cache: add[r] of them are request r's, in order."""
        stream = torch.cuda.current_stream().cuda_stream
        slots = torch.empty(len(rows), dtype=torch.int32, device="cuda")
        R.rsr_cache_slots(self.held, add, self.table, self.c.page_size, self.free, self.count, slots, self.begin, self.now, self.left, stream)
        R.rsr_cache_append(self.cache, self.k, self.v, slots, rows, stream)
        if self.left.item() < 0:
            raise RuntimeError("no page is left")
        self.held, self.now = self.now, self.held
        self.count, self.left = self.left, self.count


def draft(root: int, guesses: List[List[int]], widths: Sequence[int]):
    """(tokens, parents) of a tree: behind every token of a level the first so many guesses."""
    tokens, parents, level = [root], [-1], [0]
    for width in widths:
        below = []
        for at in level:
            for t in guesses[tokens[at]][:width]:
                below.append(len(tokens))
                tokens.append(t)
                parents.append(at)
        level = below
    return tokens, parents


def decode(model: Model, prompts: Sequence[Sequence[int]], length: int, widths: Sequence[int]) -> Dict[str, object]:
    """`length` tokens behind every prompt, with trees of these widths (none: one token at a time)."""
    if sum(np.cumprod([1, *widths])) > 64:
        raise ValueError("a tree has at most 64 tokens")
    if max(map(len, prompts)) + length + len(widths) > len(model.positions):
        raise ValueError("there is no position that far back")
    guesses = model.guesses(max(widths, default=1))
    start = [0] + np.cumsum([len(p) for p in prompts]).tolist()
    best = model.forward([t for p in prompts for t in p], start)
    model.append(torch.arange(start[-1], dtype=torch.int32).cuda(), torch.tensor([len(p) for p in prompts], dtype=torch.int32).cuda())
    found = [[t] for t in best[torch.tensor(start[1:]).cuda() - 1].tolist()]
    steps = turns = 0
    torch.cuda.synchronize()
    began = time.perf_counter()
    while min(len(f) for f in found) < length:
        trees = [draft(f[-1], guesses, widths) if len(f) < length else ([], []) for f in found]  # (who has enough has no new tokens)
        start = [0] + np.cumsum([len(t) for t, _ in trees]).tolist()
        model.forward([t for tokens, _ in trees for t in tokens], start, [p for _, parents in trees for p in parents])
        for f, more in zip(found, model.keep()):  # down the tree for as long as the model's choice was guessed
            f.extend(more)
        steps, turns = steps + 1, turns + sum(1 for t, _ in trees if t)
    torch.cuda.synchronize()
    return {"tokens": [f[:length] for f in found], "steps": steps, "seconds": time.perf_counter() - began,
            "per_step": sum(len(f) - 1 for f in found) / max(1, turns)}


def run(c: Config, requests: int, prompt: int, length: int, widths: Sequence[int]) -> Dict[str, Dict[str, object]]:
    """The same prompts one token at a time and with trees."""
    w = Weights(c)
    rng = np.random.default_rng(c.seed + 1)
    prompts = [rng.integers(0, c.vocabulary, prompt + 7 * r).tolist() for r in range(requests)]
    results = {}
    for name, tree in (("plain", ()), ("drafted", tuple(widths))):
        model = Model(c, w, requests)
        try:
            results[name] = decode(model, prompts, length, tree)
        finally:
            model.close()
    return results


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--requests", type=int, default=4)
    p.add_argument("--prompt", type=int, default=200)
    p.add_argument("--length", type=int, default=96)
    p.add_argument("--widths", type=int, nargs="*", default=[3, 2, 1], help="guesses behind a token, level by level (at most 64 tokens in a tree)")
    p.add_argument("--rotary", action="store_true", help="positions rotate normed heads, instead of embeddings of positions")
    p.add_argument("--temperature", type=float, default=0.0, help="0: the likeliest token")
    p.add_argument("--top-p", type=float, default=1.0)
    a = p.parse_args()
    results = run(Config(rotary=a.rotary, temperature=a.temperature, top_p=a.top_p), a.requests, a.prompt, a.length, a.widths)
    for name, r in results.items():
        print(f"{name:8s} {r['steps']:4d} steps, {r['per_step']:.2f} tokens per step and request, {1e3 * r['seconds'] / max(1, r['steps']):.2f} ms per step")
    print("the same tokens:", results["plain"]["tokens"] == results["drafted"]["tokens"])


if __name__ == "__main__":
    main()
