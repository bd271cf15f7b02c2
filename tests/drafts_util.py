"""Shared pieces of the drafting-step tests: batches with drafted trees, device
tensors, and tolerances.  No kernels here."""
import numpy as np
import torch

from oracle import drafts as oracle
from workloads import build_plan, make_batch
from workloads.gen import TORCH_DTYPES

# half a step relative to the value
UNIT = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}
F32 = 2.0 ** -24


def random_trees(rng, rows, spread=4, roots=1):
    """Parents of every row: `roots` rows with parent -1 first, then random ones."""
    out = []
    for n in rows:
        p = [-1 if j < roots else int(rng.integers(max(0, j - spread), j)) for j in range(n)]
        out += p
    return np.array(out, dtype=np.int32)


def tree_plan(dtype, heads, dim, groups, plen, cached, rows, parents=None, seed=0, scale=None):
    """A LayoutPlan whose own tokens are `cached` cached and `rows` drafted ones."""
    slen = [c + n for c, n in zip(cached, rows)]
    return build_plan(heads=heads, head_dim=dim, block_size=16, dtype=dtype, group_of_request=groups,
                      prefix_lens=plen, suffix_lens=slen, sm_scale=dim ** -0.5 if scale is None else scale,
                      rng=np.random.default_rng(seed), prefix_parents=parents)


def offsets_of(rows):
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)


def queries(T, heads, dim, dtype, seed=0):
    g = torch.Generator().manual_seed(seed + 1000)
    return torch.randn((T, heads, dim), generator=g).to(TORCH_DTYPES[dtype])


def out_tolerance(dtype, out, spread, noise, keys, dim):
    """Bound of |out - exact| per element.  The weights are rounded to the cache's type
    (unit u) before the products, and the output by their sum, so they enter as
    sum w |v - out| (spread); the result is rounded once (u |out|).  A logit is off by
    at most (dim + 8) 2^-24 times sum |q k| (noise), which scales its weight, as do
    the exponential and the running rescales ((16 + keys / 32) 2^-24); the fp32 sums over
    the keys add keys 2^-24 of the sum of w |v| <= |out| + spread."""
    u = UNIT[dtype]
    weight = (0.0 if dtype == "float32" else 1.02 * u) + 2.0 * F32 * ((dim + 8) * noise[..., None] + 16 + keys / 32)
    return u * np.abs(out) * 1.01 + weight * spread + (keys + 8) * F32 * (np.abs(out) + spread) + 1e-7


def lse_tolerance(lse, noise, keys, dim):
    """The logits' error, the sums' and the rounding of log2 and of the result."""
    return F32 * ((dim + 8) * noise + keys + 32 + 4 * np.abs(lse))


__all__ = ["UNIT", "F32", "random_trees", "tree_plan", "offsets_of", "queries", "out_tolerance", "lse_tolerance",
           "oracle", "make_batch", "TORCH_DTYPES"]
