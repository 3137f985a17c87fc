"""The step of a decoder between its weight products, as cases that can be timed and compared.

The products of this library (include/rsr.h) make queries, keys and values of the new tokens of a step; what stands between
them and the next product is the cache (include/rsr_cache.h): which pages and slots the requests of the step hold, the
attention of the new tokens over what their requests have in the cache and over each other (a chain: one token, or a piece of a
prompt; or a tree of drafted tokens of which one path will be kept), and the writing of the tokens that are kept.

Four operators.  "attention": softmax(scale * q . k) . v over the pages of a request and its own new tokens, whose keys and
values are rounded to the type of the cache as they will be when they are written there.  "slots": block tables, slot maps
and what is left of the free pages, from lengths.  "masks": who sees whom in drafted trees, from parents.  "append": keys
and values of kept tokens into their slots.

What varies: one request or hundreds, one new token or a piece of a prompt, caches from nothing to 131072 tokens, ragged
lengths, as many key heads as query heads (configuration 4: width 2560 as 20 heads of 128) or fewer, heads of 64 to 256,
float activations (what the products give) or 16-bit ones, caches of float16 and bfloat16, pages of 8 to 128 tokens.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LARGEST_KEYS = 4 * 131072 * 5 * 128          # values in the cached keys of the largest listed case
LARGEST_FLOPS = 4 * 64 * 20 * 4 * 128 * 131072


def listed():
    return [
        # one sequence of configuration 4 decodes one token, early on: what a call costs
        {"name": "attend_1_of_500", "what": "attention", "requests": 1, "new": 1, "held": 500, "ragged": False, "tree": False, "heads": 20, "kv_heads": 20, "dim": 128, "act": "f32", "cache": "bf16", "page": 16},
        # the sixteen vectors of configuration 4 as sixteen drafted tokens of one sequence, float activations as the products give them
        {"name": "attend_tree_16_of_4k", "what": "attention", "requests": 1, "new": 16, "held": 4096, "ragged": False, "tree": True, "heads": 20, "kv_heads": 20, "dim": 128, "act": "f32", "cache": "f16", "page": 16},
        # a served batch: ragged lengths, small trees, few key heads, 16-bit activations
        {"name": "attend_tree_ragged_32", "what": "attention", "requests": 32, "new": 16, "held": 8192, "ragged": True, "tree": True, "heads": 20, "kv_heads": 5, "dim": 128, "act": "bf16", "cache": "bf16", "page": 16},
        # nothing divides anything: heads of 80, seven requests, odd lengths, the smallest pages
        {"name": "attend_odd_80", "what": "attention", "requests": 7, "new": 13, "held": 3001, "ragged": True, "tree": True, "heads": 32, "kv_heads": 8, "dim": 80, "act": "f16", "cache": "f16", "page": 8},
        # pieces of prompts: chains of 512 new tokens behind up to 2048 that are in the cache
        {"name": "attend_chain_512", "what": "attention", "requests": 4, "new": 512, "held": 2048, "ragged": True, "tree": False, "heads": 20, "kv_heads": 20, "dim": 128, "act": "f32", "cache": "bf16", "page": 64},
        # the largest: long documents, trees of 64
        {"name": "attend_tree_64_of_128k", "what": "attention", "requests": 4, "new": 64, "held": 131072, "ragged": False, "tree": True, "heads": 20, "kv_heads": 5, "dim": 128, "act": "bf16", "cache": "bf16", "page": 64},
        # slots of a decode step: 256 requests, each keeps one to eight tokens
        {"name": "slots_step_256", "what": "slots", "requests": 256, "add": 8, "held": 8192, "page": 16},
        # slots of prompts that begin: everything is new
        {"name": "slots_prompts_64", "what": "slots", "requests": 64, "add": 16384, "held": 0, "page": 16},
        # trees: of one sequence, and of a large batch
        {"name": "masks_1", "what": "masks", "requests": 1, "new": 16},
        {"name": "masks_512", "what": "masks", "requests": 512, "new": 64},
        # the kept path of one tree of sixteen drafted tokens, and the keys and values of prompts
        {"name": "append_kept_path", "what": "append", "rows": 16, "count": 16, "keep": 0.3, "kv_heads": 20, "dim": 128, "act": "f32", "cache": "bf16", "page": 16},
        {"name": "append_prompts_16k", "what": "append", "rows": 16384, "count": 16384, "keep": 1.0, "kv_heads": 5, "dim": 128, "act": "bf16", "cache": "bf16", "page": 16},
    ]


def _between(rng, low, high):
    """A whole number between low and high, spread over its logarithm; round numbers come up too."""
    x = math.exp(rng.uniform(math.log(low), math.log(high)))
    step = rng.choice([1, 1, 1, 8, 64])
    x = int(min(high, max(low, round(x / step) * step)))
    return x - (x == 3072)


def draw(rng):
    what = rng.choice(["attention"] * 6 + ["slots", "slots", "masks", "append", "append"])
    if what == "masks":
        return {"what": what, "requests": _between(rng, 1, 1024), "new": _between(rng, 1, 64)}
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if what == "slots":
        requests = _between(rng, 1, 1024)
        if rng.random() < 0.5:
            return {"what": what, "requests": requests, "add": _between(rng, 1, 16), "held": _between(rng, 1, 32768), "page": page}
        return {"what": what, "requests": requests, "add": _between(rng, 64, max(65, min(32768, 1048576 // requests))), "held": rng.choice([0, 0, 777]), "page": page}
    cache = rng.choice(["f16", "bf16"])
    act = rng.choice(["f32", cache])
    kv_heads, dim = rng.choice([1, 2, 4, 5, 8, 8, 16, 20, 32]), rng.choice([64, 80, 112, 128, 128, 128, 160, 256])
    if what == "append":
        dim = 80 if 2 * kv_heads * dim == 3072 else dim
        rows = _between(rng, 1, 16384 * 5 * 128 // (kv_heads * dim))
        return {"what": what, "rows": rows, "count": rows, "keep": rng.choice([0.3, 0.7, 1.0]), "kv_heads": kv_heads, "dim": dim, "act": act, "cache": cache, "page": page}
    heads = kv_heads * rng.choice([g for g in (1, 1, 2, 4, 5, 8) if g * kv_heads <= 64])
    if 3072 in (kv_heads * dim, heads * dim, (heads + 2 * kv_heads) * dim):
        dim = 80
    requests, tree = _between(rng, 1, 64), rng.random() < 0.6
    new = _between(rng, 1, 64) if tree else rng.choice([1, 1, _between(rng, 1, 512)])
    held = _between(rng, 1, 131072)
    held = max(1, min(held, LARGEST_KEYS // (requests * kv_heads * dim), LARGEST_FLOPS // (4 * requests * new * heads * dim)))
    new = max(1, min(new, LARGEST_FLOPS // (8 * requests * new * heads * dim)))
    return {"what": what, "requests": requests, "new": new, "held": held, "ragged": rng.random() < 0.6, "tree": tree, "heads": heads, "kv_heads": kv_heads, "dim": dim, "act": act, "cache": cache, "page": page}


def _lengths(requests, most, ragged, least=0):
    """Lengths of the requests of a batch: all alike, or spread evenly over least .. most, in no order (the last one is `most`)."""
    if not ragged or requests == 1:
        return [most] * requests
    return [min(most, least + int((most - least + 1) * math.modf((i + 1) * 0.6180339887498949)[0])) for i in range(requests - 1)] + [most]


def _held(case):
    return _lengths(case["requests"], case["held"], case["ragged"])


def _new(case):
    return _lengths(case["requests"], case["new"], case["ragged"] and case["new"] > 1, 1)


def _trees(case):
    """Tokens of the trees of a masks case."""
    return _lengths(case["requests"], case["new"], case["new"] > 1, 1)


def _kept(case):
    """Tokens that the requests of a slots case add."""
    return _lengths(case["requests"], case["add"], True, 1)


def _held_slots(case):
    return _lengths(case["requests"], case["held"], True)


def work(case):
    what = case["what"]
    if what == "masks":
        return {"bytes": 16 * sum(_trees(case)), "flops": 0}
    if what == "slots":
        held, add, page = _held_slots(case), _kept(case), case["page"]
        pages = sum(-(-(h + a) // page) - -(-h // page) for h, a in zip(held, add))
        return {"bytes": 16 * case["requests"] + 8 * pages + 4 * sum(add), "flops": 0}
    size = 4 if case["act"] == "f32" else 2
    if what == "append":
        kept = max(1, round(case["count"] * case["keep"]))
        return {"bytes": 2 * kept * case["kv_heads"] * case["dim"] * (size + 2) + 8 * case["count"], "flops": 0}
    held, new, dim = _held(case), _new(case), case["dim"]
    cached = 2 * 2 * sum(held) * case["kv_heads"] * dim
    fresh = size * sum(new) * dim * (2 * case["heads"] + 2 * case["kv_heads"])
    pairs = sum(h * n + (n if case["tree"] else n * (n + 1) // 2) for h, n in zip(held, new))  # (a tree: at least itself)
    return {"bytes": cached + fresh + 4 * sum(-(-h // case["page"]) for h in held), "flops": 4 * dim * case["heads"] * pairs}


# ---- inputs, made on the device from the seed alone ------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(lengths):
    return torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), _ints(lengths).cumsum(0)]).to(torch.int32)


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _parents(g, new):
    """Drafted trees: a token hangs on one of those before it, most often on a late one, now and then on the cache itself (-1)."""
    index = torch.cat([torch.arange(n, device="cuda") for n in new])
    back = torch.rand(index.shape, generator=g, device="cuda").square() * (index + 1)
    return (index - 1 - back.long()).clamp(min=-1).to(torch.int32)


def _tables(g, held, page, spare=1):
    """Block tables of requests whose pages lie in no order, and the pages that are free."""
    need = [-(-h // page) for h in held]
    width, total = max(1, max(need) + spare), sum(need)
    order = torch.randperm(total + spare * len(held), generator=g, device="cuda").to(torch.int32)
    column = torch.arange(width, device="cuda")[None]
    first = (_ints(need).cumsum(0) - _ints(need))[:, None]
    table = torch.where(column < _ints(need)[:, None], order[(first + column).clamp(max=order.numel() - 1)], -1)
    return table.to(torch.int32).contiguous(), order[total:].contiguous()


def prepare(case, seed):
    g = _generator(seed)
    what = case["what"]
    if own:
        import paper_2411_06360_amd as rsr
    s = {"case": case, "stream": torch.cuda.current_stream().cuda_stream}
    if what == "masks":
        new = _trees(case)
        s.update(parent=_parents(g, new), start=_starts(new))
        s.update(mask=torch.zeros(sum(new), dtype=torch.int64, device="cuda"), depth=torch.zeros(sum(new), dtype=torch.int32, device="cuda"))
        return s
    page = case["page"]
    if what == "slots":
        held, add = _held_slots(case), _kept(case)
        table, _ = _tables(g, held, page, spare=-(-case["add"] // page) + 1)
        need = sum(-(-(h + a) // page) - -(-h // page) for h, a in zip(held, add))
        free = torch.randperm(need + need // 8 + 16, generator=g, device="cuda").to(torch.int32)
        s.update(held=_ints(held), add=_ints(add), table=table, free=free, count=_ints([free.numel()]))
        s.update(slots=torch.zeros(sum(add) + 7, dtype=torch.int32, device="cuda"), start=torch.zeros(len(held) + 1, dtype=torch.int32, device="cuda"))
        s.update(now=torch.zeros(len(held), dtype=torch.int32, device="cuda"), left=torch.zeros(1, dtype=torch.int32, device="cuda"))
        return s
    act, kind, heads, dim = DTYPES[case["act"]], DTYPES[case["cache"]], case["kv_heads"], case["dim"]
    if what == "append":
        rows, count = case["rows"], case["count"]
        pages = -(-count // page) + 3
        order = torch.randperm(pages, generator=g, device="cuda")
        place = torch.arange(count, device="cuda") + 5  # runs of slots on pages that lie in no order, from the middle of the first page on
        slots = order[place // page] * page + place % page
        kept = max(1, round(count * case["keep"]))  # behind the kept tokens the slot map says that there is nothing
        s.update(slots=torch.where(torch.arange(count, device="cuda") < kept, slots, -1).to(torch.int32))
        s.update(rows=torch.randperm(rows, generator=g, device="cuda")[:count].sort().values.to(torch.int32))
        width = 2 * heads * dim  # keys and values are parts of the rows that a product gave
        qkv = _normal(g, (rows, width), act)
        s.update(k=qkv[:, :heads * dim], v=qkv[:, heads * dim:])
        s.update(cache_k=torch.randn((pages, heads, page, dim), generator=g, device="cuda", dtype=kind), cache_v=torch.randn((pages, heads, page, dim), generator=g, device="cuda", dtype=kind))
        if own:
            s["cache"] = rsr.make_cache(s["cache_k"], s["cache_v"])
        return s
    held, new = _held(case), _new(case)
    table, free = _tables(g, held, page)
    pages = int(sum(-(-h // page) for h in held) + len(held))
    tokens, queries = sum(new), case["heads"] * dim
    qkv = _normal(g, (tokens, queries + 2 * heads * dim), act)  # the rows that the product with the q/k/v matrices gives
    qkv[:, :queries] *= 1.5
    s.update(q=qkv[:, :queries], k=qkv[:, queries:queries + heads * dim], v=qkv[:, queries + heads * dim:], out=torch.zeros((tokens, queries), dtype=act, device="cuda"))
    s.update(cache_k=torch.randn((pages, heads, page, dim), generator=g, device="cuda", dtype=kind), cache_v=torch.randn((pages, heads, page, dim), generator=g, device="cuda", dtype=kind))
    s.update(table=table, held=_ints(held), start=_starts(new), scale=dim ** -0.5)
    s["mask"] = _plain_masks(_parents(g, new), s["start"], case["new"])[0] if case["tree"] else None
    if own:
        s["cache"] = rsr.make_cache(s["cache_k"], s["cache_v"])
        s["step"] = rsr.make_step(table, s["held"], s["start"], tokens, case["new"], s["mask"])
        s["workspace"] = torch.zeros(rsr.rsr_tree_attention_workspace(s["cache"], s["step"], case["heads"]), dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------
def _padded(start, most):
    """Rows of the new tokens as [requests][most], and which of them there are."""
    index = start[:-1, None].long() + torch.arange(most, device="cuda")[None]
    there = index < start[1:, None]
    return index, there


def _twice(reach, to):
    """Reach along twice as many links: reach[r][i] is what i sees, to[r][i] the last one it sees, or i itself."""
    return reach | torch.gather(reach, 1, to[:, :, None].expand_as(reach)), torch.gather(to, 1, to)


def _plain_masks(parent, start, most):
    index, there = _padded(start, most)
    here = torch.arange(most, device="cuda")[None].expand_as(index)
    up = parent[index.clamp(max=parent.numel() - 1)].long()
    to = torch.where(there & (up >= 0) & (up < here), up, here)
    reach = here[:, :, None] == here[:, None, :]
    reach, _ = _twice(*_twice(*_twice(*_twice(*_twice(*_twice(*_twice(reach, to)))))))
    mask = (reach.long() << torch.arange(most, device="cuda")).sum(2)
    return mask[there], reach.sum(2)[there].to(torch.int32) - 1


def _plain_slots(s):
    page, table, held, add, count = s["case"]["page"], s["table"], s["held"].long(), s["add"].long(), s["count"].long()
    width, free = table.shape[1], s["free"]
    before, after = ((held + page - 1) // page).clamp(max=width), ((held + add + page - 1) // page).clamp(max=width)
    first = (after - before).cumsum(0) - (after - before)
    column = torch.arange(width, device="cuda")[None]
    taken = first[:, None] + column - before[:, None]
    page_of = torch.where(taken < count, free[(count - 1 - taken).clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where((column >= before[:, None]) & (column < after[:, None]), page_of, table))
    granted = torch.minimum((count - first).clamp(min=0), after - before)
    s["now"].copy_(torch.maximum(held, torch.minimum(held + add, (before + granted) * page)))
    s["left"].copy_(count - (after - before).sum())
    ends = add.cumsum(0)
    s["start"][1:].copy_(ends)
    token = torch.arange(s["slots"].numel(), device="cuda")
    r = torch.searchsorted(ends, token, right=True).clamp(max=held.numel() - 1)
    at = held[r] + token - (ends - add)[r]
    p = table[r, (at // page).clamp(max=width - 1)].long()
    s["slots"].copy_(torch.where((token < ends[-1]) & (p >= 0) & (at < width * page), p * page + at % page, -1))
    return {"slots": s["slots"], "table": table, "start": s["start"], "now": s["now"], "left": s["left"]}


def _plain_append(s):
    page, heads, dim = s["case"]["page"], s["case"]["kv_heads"], s["case"]["dim"]
    there = s["slots"] >= 0
    slot, row = s["slots"][there].long(), s["rows"][there].long()
    s["cache_k"][slot // page, :, slot % page] = s["k"][row].view(-1, heads, dim).to(s["cache_k"].dtype)
    s["cache_v"][slot // page, :, slot % page] = s["v"][row].view(-1, heads, dim).to(s["cache_v"].dtype)
    return {"k": s["cache_k"], "v": s["cache_v"]}


def _plain_attention(s):
    case, kind = s["case"], s["cache_k"].dtype
    requests, most, heads, kv_heads, dim = case["requests"], case["new"], case["heads"], case["kv_heads"], case["dim"]
    index, there = _padded(s["start"], most)
    row = index.clamp(max=s["q"].shape[0] - 1)

    def keys(cache, fresh):  # [requests][kv_heads][cached, then new][dim]
        old = cache[s["table"].clamp(min=0).long()].transpose(1, 2).reshape(requests, kv_heads, -1, dim)
        new = fresh[row].to(kind).view(requests, most, kv_heads, dim).transpose(1, 2)
        return torch.cat([old, new], 2).float()

    q = s["q"][row].float().view(requests, most, kv_heads, heads // kv_heads, dim).permute(0, 2, 1, 3, 4).reshape(requests, kv_heads, -1, dim)
    score = torch.matmul(q, keys(s["cache_k"], s["k"]).transpose(2, 3).contiguous()).mul_(s["scale"])
    cached = torch.arange(score.shape[3] - most, device="cuda")[None] < s["held"][:, None]
    bit = torch.arange(most, device="cuda")
    sees = (s["mask"][row][:, :, None] >> bit) & 1 == 1 if s["mask"] is not None else (bit[None, :, None] >= bit[None, None, :]).expand(requests, -1, -1)
    seen = torch.cat([cached[:, None].expand(-1, most, -1), sees & there[:, None]], 2)
    score.view(requests, kv_heads, most, heads // kv_heads, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(3, keepdim=True)
    weight = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = weight.sum(3, keepdim=True)
    out = torch.matmul(weight, keys(s["cache_v"], s["v"])) / torch.where(total == 0, 1.0, total)
    out = out.view(requests, kv_heads, most, -1, dim).permute(0, 2, 1, 3, 4).reshape(requests, most, -1)
    return out[there].to(s["q"].dtype)


def run(s):
    what = s["case"]["what"]
    if not own:
        if what == "attention":
            return _plain_attention(s)
        if what == "slots":
            return _plain_slots(s)
        if what == "append":
            return _plain_append(s)
        mask, depth = _plain_masks(s["parent"], s["start"], s["case"]["new"])
        return {"mask": mask, "depth": depth}
    import paper_2411_06360_amd as rsr

    if what == "attention":
        rsr.rsr_tree_attention(s["cache"], s["step"], s["q"], s["k"], s["v"], s["out"], s["case"]["heads"], s["scale"], s["workspace"], s["stream"])
        return s["out"]
    if what == "slots":
        rsr.rsr_cache_slots(s["held"], s["add"], s["table"], s["case"]["page"], s["free"], s["count"], s["slots"], s["start"], s["now"], s["left"], s["stream"])
        return {"slots": s["slots"], "table": s["table"], "start": s["start"], "now": s["now"], "left": s["left"]}
    if what == "append":
        rsr.rsr_cache_append(s["cache"], s["k"], s["v"], s["slots"], s["rows"], s["stream"])
        return {"k": s["cache_k"], "v": s["cache_v"]}
    rsr.rsr_tree_masks(s["parent"], s["start"], s["mask"], s["depth"], s["stream"])
    return {"mask": s["mask"], "depth": s["depth"]}


def exact(case, seed):
    """The attention by its definition in 64 bits, one request and query head at a time, and what append would write without
    rounding it; slots and masks are whole numbers."""
    if case["what"] in ("slots", "masks"):
        return None
    s = prepare(case, seed)
    if case["what"] == "append":
        kept = max(1, round(case["count"] * case["keep"]))  # (the slots behind these are -1)
        found = {}
        for name in ("k", "v"):
            flat = s["cache_" + name].double().permute(0, 2, 1, 3).reshape(-1, case["kv_heads"], case["dim"])
            flat[s["slots"][:kept].long()] = s[name].double()[s["rows"][:kept].long()].unflatten(1, (case["kv_heads"], case["dim"]))
            found[name] = flat.unflatten(0, (-1, case["page"])).permute(0, 2, 1, 3).contiguous()
        return found
    group, page, dim = case["heads"] // case["kv_heads"], case["page"], case["dim"]
    out = torch.zeros((s["q"].shape[0], case["heads"], dim), dtype=torch.float64, device="cuda")
    first = 0
    for r, (held, new) in enumerate(zip(_held(case), _new(case))):
        pages = s["table"][r, :-(-held // page)].long()
        rows = slice(first, first + new)
        if case["tree"]:
            bits = [[(m >> j) & 1 for j in range(new)] for m in s["mask"][rows].tolist()]
        else:
            bits = [[int(j <= i) for j in range(new)] for i in range(new)]
        blind = torch.tensor(bits, device="cuda").logical_not()
        for b in range(case["kv_heads"]):
            side = {}
            for name in ("k", "v"):
                old = s["cache_" + name][pages, b].reshape(-1, dim)[:held].double()
                side[name] = torch.cat([old, s[name][rows, b * dim:(b + 1) * dim].to(s["cache_" + name].dtype).double()])
            for a in range(b * group, (b + 1) * group):
                score = s["q"][rows, a * dim:(a + 1) * dim].double() @ side["k"].T.contiguous() * s["scale"]
                score[:, held:].masked_fill_(blind, -math.inf)
                weight = torch.softmax(score, 1).nan_to_num(0.0)
                out[rows, a] = weight @ side["v"]
        first += new
    return out.view(-1, case["heads"] * dim)
