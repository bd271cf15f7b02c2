"""Shared pieces of the tests of caches held in 8 bits: pools of a batch, calls, bounds.
No kernels here."""
import numpy as np
import torch

import drafts_util as du
from drafts_util import oracle as drafts_oracle
from gpu_util import problem_for
from oracle import cache8 as oracle

INTS = ("prefix_tables", "prefix_lens", "prefix_parents", "suffix_tables", "suffix_lens", "group_ids")


def pools_of(batch, loud=None):
    """(device pools, dense float64 keys and values) of a batch's cache quantised; slots that
    hold no token are NaN codes.  loud: factors [heads] on the values."""
    out, dense = {}, []
    for name, x in (("k", batch.k_pool), ("v", batch.v_pool)):
        x = x.double().numpy()
        if loud is not None and name == "v":
            x = x * np.asarray(loud)[None, :, None, None]
        codes, byte = oracle.pack(x)
        dense.append(oracle.values(codes, byte))
        out[name] = codes if name == "k" else oracle.value_order(codes)
        out["s" + name] = byte
    return device_pools(out["k"], out["v"], np.stack([out["sk"], out["sv"]], -1)), dense


def device_pools(k, v, scales, device="cuda"):
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(device)
    return {"k": t(k).view(torch.float8_e4m3fn), "v": t(v).view(torch.float8_e4m3fn),
            "scales": t(scales).view(torch.float8_e8m0fnu)}


def ints_of(batch, off, device="cuda"):
    t = {k: torch.from_numpy(np.ascontiguousarray(v)).to(device) for k, v in batch.int_arrays().items() if v is not None}
    t["query_offsets"] = torch.from_numpy(np.ascontiguousarray(off)).to(device)
    return t


def handles(plan, off, ratio, T=None, **counts):
    import paper_2405_19888_amd as parrot
    rows = parrot.tree_rows_from_host(off, plan.group_ids, plan.num_groups, plan.heads * ratio,
                                      plan.prefix_parents if plan.nested else None)
    rows.num_query_rows = int(off[-1]) if T is None else T
    for k, v in counts.items():
        setattr(rows, k, v)
    planner = parrot.Cache8Planner(problem_for(plan), rows, nested=plan.nested)
    return planner, parrot.Cache8Decoder(planner)


def poison(planner, dec):
    planner.plan.fill_(0x7fffffff)
    dec.out.fill_(float("nan"))
    dec.lse.fill_(float("nan"))
    dec.workspace.fill_(0xFF)


def run(plan, batch, pools, q, off, T=None, check_inputs=True):
    """One plan and call on poisoned buffers; (out, lse, planner, decoder, device tensors)."""
    import paper_2405_19888_amd as parrot
    t = ints_of(batch, off)
    t["q_rows"], t["prefix"], t["suffix"] = q.cuda(), pools, pools
    planner, dec = handles(plan, off, q.shape[1] // plan.heads, q.shape[0] if T is None else T)
    if check_inputs:
        parrot.parrot_validate_cache8_inputs(
            planner.problem, planner.rows, t["query_offsets"], t["prefix_tables"], t["prefix_lens"],
            t["prefix_parents"] if plan.nested else None, t["suffix_tables"], t["suffix_lens"], t["group_ids"],
            torch.zeros(16, dtype=torch.int32, device="cuda"))
    poison(planner, dec)
    planner(t)
    dec(t)
    torch.cuda.synchronize()
    return dec.out, dec.lse, planner, dec, t


def reference(plan, dense, q, off):
    return drafts_oracle.shared_prefix_tree(
        q, off, None, dense[0], dense[1], dense[0], dense[1], plan.prefix_tables, plan.prefix_lens, plan.suffix_tables,
        plan.suffix_lens, plan.group_ids, plan.sm_scale, plan.prefix_parents if plan.nested else None)


def check(plan, dense, q, off, out, lse, what=""):
    """As the tree calls' bounds: float32 operands come in three parts, whose products are
    summed as three times the elements."""
    ref, rlse, spread, noise = reference(plan, dense, q, off)
    n = int(off[-1])
    dim = plan.head_dim * (3 if plan.dtype == "float32" else 1)
    keys = int(plan.suffix_lens.max()) + int(plan.prefix_lens.sum() if plan.nested else max([0] + list(plan.prefix_lens)))
    got, glse = out.double().cpu().numpy()[:n], lse.double().cpu().numpy()[:n]
    tol = du.out_tolerance(plan.dtype, ref[:n], spread[:n], noise[:n], keys, dim)
    ltol = du.lse_tolerance(rlse[:n], noise[:n], keys, dim)
    assert np.isfinite(got).all() and np.isfinite(glse).all(), what
    worst = (np.abs(got - ref[:n]) / tol).max()
    lworst = (np.abs(glse - rlse[:n]) / ltol).max()
    print(f"{what}: out error {worst:.2f} of its bound, lse {lworst:.2f}", flush=True)
    assert worst <= 1.0 and lworst <= 1.0, (what, worst, lworst)
    assert torch.isnan(out[n:]).all() and torch.isnan(lse[n:]).all(), "padding rows were written"


__all__ = ["oracle", "du", "drafts_oracle", "pools_of", "device_pools", "ints_of", "handles", "poison", "run", "reference",
           "check", "problem_for"]
