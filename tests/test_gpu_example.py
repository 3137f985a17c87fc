"""examples/tree_decode.py: the operators together decode what a plain model in float64 decodes, with trees as without."""
import numpy as np
import pytest

from examples.tree_decode import Config, Weights, run

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16().double().numpy()


def plain_decode(c: Config, w: Weights, prompt, length):
    """The likeliest tokens one by one in float64 (keys and values rounded as the cache rounds them), and by how much the closest
    decision was won."""
    m = {n: a.astype(np.float64) * w.scale for n, a in w.matrices.items()}
    group, d = c.heads // c.kv_heads, c.head_dim
    keys, values, found, closest = [], [], [], np.inf
    tokens = list(prompt)
    for at in range(len(prompt) + length - 1):
        x = w.tokens[tokens[at]].astype(np.float64) + w.positions[at]
        keys.append(bf16(x @ m["k"]).reshape(c.kv_heads, d))
        values.append(bf16(x @ m["v"]).reshape(c.kv_heads, d))
        if at < len(prompt) - 1:
            continue
        q, K, V = (x @ m["q"]).reshape(c.heads, d), np.array(keys), np.array(values)
        mixed = np.empty((c.heads, d))
        for a in range(c.heads):
            s = K[:, a // group] @ q[a] * d ** -0.5
            e = np.exp(s - s.max())
            mixed[a] = e @ V[:, a // group] / e.sum()
        scores = (x + w.attention * (mixed.reshape(-1) @ m["o"])) @ m["head"]
        first, second = np.sort(scores)[:-3:-1]
        closest = min(closest, first - second)
        tokens.append(int(scores.argmax()))
    return tokens[len(prompt):], closest


@pytest.mark.parametrize("widths", [(3, 2, 1), (1,), (4, 4)])
def test_trees_decode_what_single_tokens_do(widths):
    print("example", widths, flush=True)
    c = Config(hidden=256, heads=4, kv_heads=2, vocabulary=64, k=6, page_size=16, pages=48, pages_per_request=8, seed=3)
    results = run(c, requests=3, prompt=5, length=40, widths=widths)
    assert results["plain"]["tokens"] == results["drafted"]["tokens"]
    assert results["plain"]["per_step"] == 1.0 and results["drafted"]["per_step"] >= 1.0
    assert results["drafted"]["steps"] <= results["plain"]["steps"]
    rng, w = np.random.default_rng(c.seed + 1), Weights(c)
    for r in range(3):
        prompt = rng.integers(0, c.vocabulary, 5 + 7 * r).tolist()
        wanted, closest = plain_decode(c, w, prompt, 40)
        got = results["drafted"]["tokens"][r]
        # a decision won by less than float's error, or a key on the edge of a rounding of the cache, may fall otherwise: then up to there
        assert closest > 1e-2, "the seed has a close decision"
        assert got == wanted
