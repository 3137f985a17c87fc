"""What a decoder's step does on both sides of its attention, as cases that can be timed and compared.

The products of this library give queries and keys without positions, and behind the last product scores of the next tokens.
Three operators (include/rsr_decode.h) make a step of them that never leaves the device:

"rotate": norms of the queries' and keys' heads and the rotation by the tokens' positions, in one pass over the rows that the
q/k/v products gave, into rows of the type that the attention takes.  "sample": a token for every row of scores, with temperature,
top-k, top-p and min-p, each row its own, from given random numbers.  "keep": the path of a drafted tree that the chosen tokens
agree with, as the rows, counts and tokens that the cache's operators and the next step take.

What varies: one token to prompts of thousands, heads of 64 to 256 rotated in whole or in part, with norms and without, halves or
neighbours as pairs, positions up to a million, every pairing of types; one row of scores to a thousand, vocabularies of some dozen
to a quarter of a million tokens, peaked and flat scores, 16-bit scores with many equal ones; one tree to a thousand.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LARGEST_ROWS = 16384 * 25 * 128   # values of the largest listed rotation
LARGEST_SCORES = 256 * 131072     # of the largest listed rows of scores


def listed():
    return [
        # one sequence of configuration 4 (width 2560 as 20 heads of 128) decodes one token: what a call costs
        {"name": "rotate_1", "what": "rotate", "tokens": 1, "heads": 20, "kv_heads": 20, "dim": 128, "rotated": 128, "norm": True, "pairs": False, "act": "f32", "out": "f32", "far": 500},
        # nothing is round: heads of 80 of which half is rotated, neighbours as pairs, no norm, 16-bit rows, far positions
        {"name": "rotate_odd_80", "what": "rotate", "tokens": 91, "heads": 32, "kv_heads": 8, "dim": 80, "rotated": 40, "norm": False, "pairs": True, "act": "f16", "out": "f16", "far": 1000000},
        # a served batch: 32 trees of 16 drafted tokens, few key heads, float rows as the products give them, 16-bit ones for the attention
        {"name": "rotate_trees_512", "what": "rotate", "tokens": 512, "heads": 20, "kv_heads": 5, "dim": 128, "rotated": 128, "norm": True, "pairs": False, "act": "f32", "out": "bf16", "far": 8192},
        # the largest: pieces of prompts
        {"name": "rotate_prompts_16k", "what": "rotate", "tokens": 16384, "heads": 20, "kv_heads": 5, "dim": 128, "rotated": 128, "norm": True, "pairs": False, "act": "f32", "out": "bf16", "far": 131072},
        # one sequence decodes one token
        {"name": "sample_1_of_32k", "what": "sample", "rows": 1, "columns": 32768, "act": "f32", "peak": 8.0, "temperature": 0.8, "top_k": 50, "top_p": 0.9, "min_p": 0.0, "mixed": False},
        # a tree of sixteen drafted tokens, a large vocabulary, the likeliest that make up 95 %
        {"name": "sample_tree_16", "what": "sample", "rows": 16, "columns": 131072, "act": "f32", "peak": 8.0, "temperature": 1.0, "top_k": 0, "top_p": 0.95, "min_p": 0.0, "mixed": False},
        # 16-bit scores, of which many are equal, a vocabulary that nothing divides, everything at once
        {"name": "sample_odd_37", "what": "sample", "rows": 37, "columns": 50021, "act": "bf16", "peak": 6.0, "temperature": 0.7, "top_k": 40, "top_p": 0.9, "min_p": 0.05, "mixed": False},
        # hot: flat scores, tens of thousands of tokens make up 98 %
        {"name": "sample_hot_64", "what": "sample", "rows": 64, "columns": 100000, "act": "f16", "peak": 0.0, "temperature": 1.5, "top_k": 0, "top_p": 0.98, "min_p": 0.0, "mixed": False},
        # the largest: a served batch whose requests all ask for something else
        {"name": "sample_batch_256", "what": "sample", "rows": 256, "columns": 131072, "act": "f32", "peak": 8.0, "temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, "mixed": True},
        # trees: of one sequence, and of a large batch
        {"name": "keep_1", "what": "keep", "requests": 1, "new": 16, "right": 0.8, "chain": False},
        {"name": "keep_512", "what": "keep", "requests": 512, "new": 64, "right": 0.8, "chain": False},
    ]


def _between(rng, low, high):
    """A whole number between low and high, spread over its logarithm; round numbers come up too."""
    x = math.exp(rng.uniform(math.log(low), math.log(high)))
    step = rng.choice([1, 1, 1, 8, 64])
    return int(min(high, max(low, round(x / step) * step)))


def draw(rng):
    what = rng.choice(["rotate"] * 3 + ["sample"] * 4 + ["keep"] * 2)
    if what == "keep":
        return {"what": what, "requests": _between(rng, 1, 1024), "new": _between(rng, 1, 64), "right": rng.choice([0.3, 0.8, 0.95]), "chain": rng.random() < 0.3}
    act = rng.choice(["f32", "f32", "f16", "bf16"])
    if what == "rotate":
        kv_heads, dim = rng.choice([1, 2, 4, 5, 8, 8, 16, 20, 32]), rng.choice([64, 80, 112, 128, 128, 128, 160, 256])
        heads = kv_heads * rng.choice([g for g in (1, 1, 2, 4, 5, 8) if g * kv_heads <= 64])
        rotated = rng.choice([dim, dim, dim // 2 // 8 * 8])
        return {"what": what, "tokens": _between(rng, 1, min(16384, LARGEST_ROWS // ((heads + kv_heads) * dim))), "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotated": rotated,
                "norm": rng.random() < 0.7, "pairs": rng.random() < 0.3, "act": act, "out": rng.choice([act, "f32", "f16", "bf16"]), "far": _between(rng, 1, 1000000)}
    columns = _between(rng, 64, 262144)
    return {"what": what, "rows": _between(rng, 1, min(1024, LARGEST_SCORES // columns)), "columns": columns, "act": act, "peak": rng.choice([0.0, 4.0, 8.0, 12.0]),
            "temperature": rng.choice([0.0, 0.3, 0.7, 1.0, 1.0, 1.5]), "top_k": rng.choice([0, 0, 1, 20, 50, 1000, 5000]), "top_p": rng.choice([1.0, 0.5, 0.9, 0.95, 0.99]),
            "min_p": rng.choice([0.0, 0.0, 0.05, 0.2]), "mixed": rng.random() < 0.3}


def _lengths(requests, most):
    """Tokens of the trees: spread evenly over 1 .. most, in no order (the last one has `most`)."""
    return [min(most, 1 + int(most * math.modf((i + 1) * 0.6180339887498949)[0])) for i in range(requests - 1)] + [most]


def work(case):
    if case["what"] == "keep":
        tokens = sum(_lengths(case["requests"], case["new"]))
        return {"bytes": (16 if case["chain"] else 20) * tokens + 12 * case["requests"], "flops": 0}
    size = 4 if case["act"] == "f32" else 2
    if case["what"] == "rotate":
        values = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": values * (size + (4 if case["out"] == "f32" else 2)) + 4 * case["tokens"], "flops": values * (7 if case["norm"] else 3)}
    values = case["rows"] * case["columns"]
    return {"bytes": values * size + 32 * case["rows"], "flops": 4 * values}


# ---- inputs, made on the device from the seed alone ------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _zeros(shape, dtype):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def _uniform(g, shape):
    return torch.rand(shape, generator=g, device="cuda")


def _rows_of(value, rows, dtype):
    return torch.full((rows,), value, dtype=dtype, device="cuda")


def _prepare_rotate(s, case, g):
    tokens, heads, kv_heads, dim = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    # the rows that the products with the q/k/v matrices give, values among them
    qkv = (torch.randn((tokens, (heads + 2 * kv_heads) * dim), generator=g, device="cuda") * 3.0).to(DTYPES[case["act"]])
    s.update(q=qkv[:, :heads * dim], k=qkv[:, heads * dim:(heads + kv_heads) * dim], position=torch.randint(0, case["far"] + 1, (tokens,), generator=g, device="cuda", dtype=torch.int32))
    half = case["rotated"] // 2
    s["frequency"] = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    s["eps"] = 1e-6 if case["norm"] else None
    for name in ("q_weight", "k_weight"):
        s[name] = 1.0 + 0.2 * torch.randn(dim, generator=g, device="cuda") if case["norm"] else None
    s.update(q_out=_zeros((tokens, heads * dim), DTYPES[case["out"]]), k_out=_zeros((tokens, kv_heads * dim), DTYPES[case["out"]]))
    if own:
        import paper_2411_06360_amd as rsr

        s["rotary"] = rsr.make_rotary(s["frequency"], dim, eps=s["eps"], q_weight=s["q_weight"], k_weight=s["k_weight"], pairs=case["pairs"])


def _prepare_sample(s, case, g):
    rows, columns = case["rows"], case["columns"]
    logits = torch.randn((rows, columns), generator=g, device="cuda") * 2.0
    if case["peak"]:  # a few tokens stand out, most of them a little
        few = max(1, min(64, columns // 4))
        at = torch.randint(0, columns, (rows, few), generator=g, device="cuda")
        logits.scatter_add_(1, at, case["peak"] * _uniform(g, (rows, few)).square() + 2.0)
    s["logits"] = logits.to(DTYPES[case["act"]])
    s["uniform"] = _uniform(g, (rows,))
    if case["mixed"]:  # greedy, top-k, top-p, min-p, all of them, temperature alone: request by request
        kind = torch.arange(rows, device="cuda") % 6
        pick = torch.tensor([[0.0, 0.8, 1.0, 1.0, 0.7, 1.0], [0, 50, 0, 0, 40, 0], [1.0, 1.0, 0.9, 1.0, 0.95, 1.0], [0.0, 0.0, 0.0, 0.1, 0.02, 0.0]], device="cuda")[:, kind]
        s.update(temperature=pick[0].contiguous(), top_k=pick[1].to(torch.int32), top_p=pick[2].contiguous(), min_p=pick[3].contiguous())
    else:
        s.update(temperature=_rows_of(case["temperature"], rows, torch.float32), top_k=_rows_of(case["top_k"], rows, torch.int32),
                 top_p=_rows_of(case["top_p"], rows, torch.float32), min_p=_rows_of(case["min_p"], rows, torch.float32))
    s.update(token=_zeros(rows, torch.int32), probability=_zeros(rows, torch.float32), kept=_zeros(rows, torch.int32))
    if own:
        import paper_2411_06360_amd as rsr

        s["workspace"] = _zeros(rsr.rsr_sample_workspace(rows, columns), torch.uint8)


def _prepare_keep(s, case, g):
    new = _lengths(case["requests"], case["new"])
    index = torch.cat([torch.arange(n, device="cuda") for n in new])
    begin = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), _ints(new).cumsum(0)])
    # a token hangs on one of those before it, most often on a late one; now and then a guess behind the cache itself (-1)
    parent = index - 1 if case["chain"] else (index - 1 - (_uniform(g, index.shape).square() * (index + 1)).long()).clamp(min=-1)
    drafted = torch.randint(0, 32000, index.shape, generator=g, device="cuda", dtype=torch.int32)
    # what is chosen behind a token is what the last of its good guesses says, and else something else
    here = begin[:-1].repeat_interleave(_ints(new).long()) + parent
    right = (_uniform(g, index.shape) < case["right"]) & (parent >= 0)
    guess = torch.where(right, torch.arange(index.numel(), device="cuda"), -1)
    guess = torch.full_like(index, -1).scatter_reduce(0, here.clamp(min=0), guess, "amax")
    chosen = torch.randint(0, 32000, index.shape, generator=g, device="cuda", dtype=torch.int32)
    chosen = torch.where(guess >= 0, drafted[guess.clamp(min=0)], chosen)
    s.update(drafted=drafted, chosen=chosen, parent=None if case["chain"] else parent.to(torch.int32), start=begin.to(torch.int32))
    tokens = sum(new)
    s.update(rows=_zeros(tokens, torch.int32), found=_zeros(tokens, torch.int32), add=_zeros(len(new), torch.int32), first=_zeros(len(new) + 1, torch.int32))


def prepare(case, seed):
    s = {"case": case, "stream": torch.cuda.current_stream().cuda_stream}
    {"rotate": _prepare_rotate, "sample": _prepare_sample, "keep": _prepare_keep}[case["what"]](s, case, _generator(seed))
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------
def _plain_heads(s, x, weight, out):
    case, rotated = s["case"], s["case"]["rotated"]
    x = x.float().unflatten(1, (-1, case["dim"]))
    if case["norm"]:
        x = x * torch.rsqrt(x.square().mean(2, keepdim=True) + s["eps"]) * weight
    angle = s["position"].double()[:, None, None] * s["frequency"]  # (in 64 bits: a far position has few bits left behind the point)
    cos, sin = angle.cos().float(), angle.sin().float()
    turned, rest = x[..., :rotated], x[..., rotated:]
    if case["pairs"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], 3).flatten(2)
    else:
        a, b = turned[..., :rotated // 2], turned[..., rotated // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], 2)
    return torch.cat([turned, rest], 2).flatten(1).to(out.dtype)


def _plain_sample(s):
    """The rows sorted, then sums in 64 bits: next to a border of a sum over a vocabulary 32 bits choose another token."""
    logits = s["logits"].float()
    columns = logits.shape[1]
    value, order = torch.sort(logits, dim=1, descending=True, stable=True)
    temperature, top_p, min_p, uniform = (s[name].double()[:, None] for name in ("temperature", "top_p", "min_p", "uniform"))
    top_k = s["top_k"].long()[:, None]
    greedy = temperature <= 0
    weight = torch.exp((value.double() - value[:, :1].double()) / torch.where(greedy, 1.0, temperature))
    top_k = torch.where(greedy, 1, torch.where((top_k <= 0) | (top_k > columns), columns, top_k))
    total = weight.cumsum(1)
    mass = total.gather(1, top_k - 1)
    nucleus = torch.where(top_p < 1, (total < top_p * mass).sum(1, keepdim=True) + 1, columns)
    likely = (weight >= min_p).sum(1, keepdim=True)
    kept = torch.minimum(torch.minimum(top_k, nucleus), likely.clamp(min=1))
    mass = total.gather(1, kept - 1)
    at = torch.minimum((total <= uniform * mass).sum(1, keepdim=True), kept - 1)
    return {"token": order.gather(1, at)[:, 0].to(torch.int32), "probability": (weight.gather(1, at) / mass)[:, 0].float(), "kept": kept[:, 0].to(torch.int32)}


def _plain_keep(s):
    most, start = s["case"]["new"], s["start"].long()
    index = start[:-1, None] + torch.arange(most, device="cuda")[None]
    there = index < start[1:, None]
    index = index.clamp(max=s["drafted"].numel() - 1)
    here = torch.arange(most, device="cuda")[None].expand_as(index)
    parent = here - 1 if s["parent"] is None else s["parent"][index].long()
    up = parent.clamp(min=0)
    right = there & (parent >= 0) & (parent < here) & (s["drafted"][index] == s["chosen"][index].gather(1, up))
    # of two guesses behind one token that say the same the first one counts
    twin = right[:, :, None] & right[:, None, :] & (parent[:, :, None] == parent[:, None, :]) & (here[:, :, None] < here[:, None, :])
    to = torch.where(right & ~twin.any(1), up, torch.where(here == 0, 0, most))  # token `most`: not on the path
    to = torch.cat([to, torch.full_like(to[:, :1], most)], 1)
    to = to.gather(1, to)
    to = to.gather(1, to)
    to = to.gather(1, to)
    to = to.gather(1, to)
    to = to.gather(1, to)
    to = to.gather(1, to)  # where 64 links lead: to token 0 from what is on the path
    on = there & (to[:, :most] == 0)
    add = on.sum(1)
    first = torch.cat([torch.zeros_like(add[:1]), add.cumsum(0)])
    place = torch.where(on, first[:-1, None] + on.cumsum(1) - 1, s["rows"].numel())
    rows = torch.full((s["rows"].numel() + 1,), -1, dtype=torch.int32, device="cuda").scatter(0, place.flatten(), index.flatten().to(torch.int32))[:-1]
    found = torch.where(rows >= 0, s["chosen"][rows.clamp(min=0).long()], -1)
    return {"rows": rows, "found": found, "add": add.to(torch.int32), "first": first.to(torch.int32)}


def run(s):
    case = s["case"]
    if not own:
        if case["what"] == "rotate":
            return {"q": _plain_heads(s, s["q"], s["q_weight"], s["q_out"]), "k": _plain_heads(s, s["k"], s["k_weight"], s["k_out"])}
        return _plain_sample(s) if case["what"] == "sample" else _plain_keep(s)
    import paper_2411_06360_amd as rsr

    if case["what"] == "rotate":
        rsr.rsr_head_rotate(s["rotary"], s["q"], s["k"], s["position"], s["q_out"], s["k_out"], s["stream"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if case["what"] == "sample":
        rsr.rsr_sample(s["logits"], s["uniform"], s["token"], s["workspace"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                       probability=s["probability"], kept=s["kept"], stream=s["stream"])
        return {"token": s["token"], "probability": s["probability"], "kept": s["kept"]}
    rsr.rsr_tree_keep(s["drafted"], s["chosen"], s["parent"], s["start"], s["rows"], s["found"], s["add"], s["first"], s["stream"])
    return {"rows": s["rows"], "found": s["found"], "add": s["add"], "first": s["first"]}


def exact(case, seed):
    """Rotations as products of complex numbers in 64 bits, and the probabilities of the sampled tokens, row by row from the
    definition; tokens, counts and paths are whole numbers."""
    if case["what"] == "keep":
        return None
    s = prepare(case, seed)
    if case["what"] == "rotate":
        half, dim, found = case["rotated"] // 2, case["dim"], {}
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(s["position"].double(), s["frequency"]))
        first = torch.arange(half, device="cuda") * (2 if case["pairs"] else 1)
        second = first + (1 if case["pairs"] else half)
        for name in ("q", "k"):
            x = s[name].double().view(case["tokens"], -1, dim).clone()
            for head in range(x.shape[1]):
                h = x[:, head]
                if case["norm"]:
                    h = h / ((h * h).sum(1, keepdim=True) / dim + s["eps"]).sqrt() * s[name + "_weight"].double()
                z = torch.complex(h[:, first], h[:, second]) * turn
                h = h.clone()
                h[:, first], h[:, second] = z.real, z.imag
                x[:, head] = h
            found[name] = x.flatten(1)
        return found
    probability = []
    for r in range(case["rows"]):
        x = s["logits"][r].double().cpu()
        t, k, p, m, u = (float(s[name][r]) for name in ("temperature", "top_k", "top_p", "min_p", "uniform"))
        if t <= 0:
            probability.append(1.0)
            continue
        x = (x - x.max()) / t
        n = int(k) if 0 < k <= case["columns"] else case["columns"]
        weight = torch.topk(x, n).values.exp().numpy()  # (of equal ones it does not matter which: their weights are the same)
        if p < 1:
            weight = weight[:int((weight.cumsum() < p * weight.sum()).sum()) + 1]
        weight = weight[:max(1, int((weight >= m).sum()))]
        at = min(int((weight.cumsum() <= u * weight.sum()).sum()), len(weight) - 1)
        probability.append(float(weight[at] / weight.sum()))
    return {"token": None, "kept": None, "probability": torch.tensor(probability, dtype=torch.float64, device="cuda")}
