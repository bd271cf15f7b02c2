"""Every kernel that a tree call may take, by type, head size and columns: which one runs,
parity over nested prefixes and real trees with several steps a wave, and what drafted
tokens hold that a row does not see."""
import ctypes

import numpy as np
import pytest
import torch

import drafts_util as du
from drafts_util import oracle
from gpu_util import problem_for
from test_tree_gpu import check, run

pytestmark = pytest.mark.gpu

TYPES = [("float16", 128), ("float16", 64), ("bfloat16", 128), ("bfloat16", 64), ("float32", 128), ("float32", 64)]
COLUMNS = {"16": 8, "32": 16, "more": 37}              # rows of the longest tree, two query heads each
PATHS = {"one": 0, "split": 1}


def kernel_of(dtype, dim, columns, path):
    """The kernel as parrot_test_tree_kernel names it."""
    few = columns == "16"
    if path == "one":                                  # rows of 256 bytes and more are shared by waves
        return 1 if few and (dim == 128 or dtype == "float32") else 0
    if columns == "32" and dtype != "float32":
        return 4
    return 3 if few else 2


@pytest.fixture(params=["one", "split"])
def path(request):
    import paper_2405_19888_amd as parrot
    force = parrot.load_library().parrot_test_tree_path
    force(PATHS[request.param])
    yield request.param
    force(-1)


def batch_of(dtype, dim, columns, seed):
    """Three requests on chains of four, one and no prefixes, drafted tokens at odd offsets."""
    most = COLUMNS[columns]
    rows, cached = [most, max(1, most - 3), most], [1203, 45, 310]
    plan = du.tree_plan(dtype, 2, dim, [3, 0, -1], [130, 33, 70, 45], cached, rows, [-1, 0, 1, 2], seed=seed)
    up = du.random_trees(np.random.default_rng(seed + 50), rows, spread=4, roots=2)
    off = du.offsets_of(rows)
    return plan, du.make_batch(plan, seed=seed), off, up, du.queries(int(off[-1]) + 2, 4, dim, dtype, seed=seed), rows, cached


def takes(dec, plan):
    import paper_2405_19888_amd as parrot
    return parrot.load_library().parrot_test_tree_kernel(ctypes.byref(dec.problem), ctypes.byref(dec.rows), int(plan.nested))


@pytest.mark.parametrize("columns", COLUMNS)
@pytest.mark.parametrize("dtype,dim", TYPES)
def test_parity(path, dtype, dim, columns):
    plan, batch, off, up, q, _, _ = batch_of(dtype, dim, columns, seed=len(columns) + dim)
    out, lse, dec, _ = run(plan, batch, q, off, up)
    assert takes(dec, plan) == kernel_of(dtype, dim, columns, path)
    check(plan, batch, q, off, up, out, lse, what=f"{path} {dtype} {dim} columns {columns}")


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("columns", COLUMNS)
@pytest.mark.parametrize("dtype,dim", TYPES)
def test_masked_tokens_hold_anything(path, dtype, dim, columns, value):
    """Drafted tokens whose values (one element of a head, neighbouring tokens, the last one
    whole) and then whose keys are no finite numbers: rows that do not see them keep every
    bit, rows that do get them where they stand."""
    plan, batch, off, up, q, rows, cached = batch_of(dtype, dim, columns, seed=3)
    clean, clse, dec, _ = run(plan, batch, q, off, up)
    assert takes(dec, plan) == kernel_of(dtype, dim, columns, path)
    n, last = int(off[-1]), rows[0] - 1
    held = {(0, 2): [5], (0, 3): [5, dim - 1], (0, last): list(range(dim)), (2, 0): [17]}    # (request, token): elements
    slot = lambda r, t: (int(plan.suffix_tables[r][(cached[r] + t) // 16]), (cached[r] + t) % 16)
    hits = torch.zeros((n, dim), dtype=torch.bool)                             # by query heads 2, 3
    sees = torch.zeros(n, dtype=torch.bool)
    for (r, t), elements in held.items():
        blk, at = slot(r, t)
        batch.v_pool[blk, 1, at, elements] = value
        for j in range(rows[r]):
            if t in oracle.tree_path(up[off[r]:off[r + 1]], j):
                hits[int(off[r]) + j, elements] = True
                sees[int(off[r]) + j] = True
    assert sees.any() and not sees.all()
    got, glse, _, _ = run(plan, batch, q, off, up)
    got, clean = got[:n].cpu(), clean[:n].cpu()
    assert torch.equal(glse[:n], clse[:n])
    assert torch.equal(got[:, :2], clean[:, :2])
    for head in (2, 3):
        assert torch.equal(got[:, head][~hits], clean[:, head][~hits])
        hit = got[:, head][hits]
        assert torch.isnan(hit).all() if value != value else (hit == value).all()
    for r, t in held:
        blk, at = slot(r, t)
        batch.k_pool[blk, 1, at, :] = value
    got, glse, _, _ = run(plan, batch, q, off, up)
    got, glse = got[:n].cpu(), glse[:n].cpu()
    assert torch.equal(got[~sees], clean[~sees]) and torch.equal(glse[~sees], clse[:n].cpu()[~sees])
    assert torch.equal(got[:, :2], clean[:, :2])


@pytest.mark.parametrize("columns", COLUMNS)
@pytest.mark.parametrize("dtype,dim", TYPES)
def test_logits_that_are_no_finite_numbers(path, dtype, dim, columns):
    """Queries of infinities and NaN, and logits that are all -inf, give NaN in output and
    lse on every kernel; single logits of -inf are weights of 0; other rows keep every bit."""
    plan, batch, off, up, q, rows, cached = batch_of(dtype, dim, columns, seed=7)
    q = q.abs() + 0.125
    clean, clse, dec, _ = run(plan, batch, q, off, up)
    assert takes(dec, plan) == kernel_of(dtype, dim, columns, path)
    n = int(off[-1])
    clean, clse = clean[:n].cpu(), clse[:n].cpu()
    x = q.clone()
    x[0, 1], x[2, 3], x[n - 1] = float("inf"), float("nan"), -float("inf")
    got, glse, _, _ = run(plan, batch, x, off, up)
    got, glse = got[:n].cpu(), glse[:n].cpu()
    bad = torch.zeros((n, 4), dtype=torch.bool)
    bad[0, 1] = bad[2, 3] = bad[n - 1] = True
    assert torch.isnan(got[bad]).all() and torch.isnan(glse[bad]).all()
    assert torch.equal(got[~bad], clean[~bad]) and torch.equal(glse[~bad], clse[~bad])

    # request 2 has no prefix: the keys of its cached tokens, then all its keys, in cache head 1
    def clear(lo, hi):
        for p in range(lo, hi):
            batch.k_pool[int(plan.suffix_tables[2][p // 16]), 1, p % 16] = -float("inf")
    clear(0, cached[2])
    got, glse, _, _ = run(plan, batch, q, off, up)
    got, glse = got[:n].cpu(), glse[:n].cpu()
    mine = torch.zeros((n, 4), dtype=torch.bool)
    mine[int(off[2]):, 2:] = True
    assert torch.equal(got[~mine], clean[~mine]) and torch.equal(glse[~mine], clse[~mine])
    ref, rlse, spread, _ = oracle.shared_prefix_tree(
        q, off, up, batch.k_pool, batch.v_pool, batch.k_pool, batch.v_pool, plan.prefix_tables, plan.prefix_lens,
        plan.suffix_tables, plan.suffix_lens, plan.group_ids, plan.sm_scale, plan.prefix_parents)
    finite = batch.k_pool.double()
    finite = float(finite[finite.isfinite()].abs().max())
    noise = plan.sm_scale * finite * q[:n].double().abs().sum(-1).numpy()          # no logit has more
    tol = du.out_tolerance(dtype, ref[:n], spread[:n], noise, cached[2] + rows[2], dim)
    ltol = du.lse_tolerance(rlse[:n], noise, cached[2] + rows[2], dim)
    at = mine.numpy()
    assert (np.abs(got.double().numpy() - ref[:n])[at] <= tol[at]).all()
    assert (np.abs(glse.double().numpy() - rlse[:n])[at] <= ltol[at]).all()
    clear(cached[2], cached[2] + rows[2])
    got, glse, _, _ = run(plan, batch, q, off, up)
    got, glse = got[:n].cpu(), glse[:n].cpu()
    assert torch.isnan(got[mine]).all() and torch.isnan(glse[mine]).all()
    assert torch.equal(got[~mine], clean[~mine]) and torch.equal(glse[~mine], clse[~mine])


def test_one_workspace_serves_smaller_batches():
    """A workspace sized for the largest batch, which takes one launch, holds the partial
    results of a part of it, which does not."""
    import paper_2405_19888_amd as parrot
    rows, cached = [64] * 16, [936 - 7 * r for r in range(16)]
    plan = du.tree_plan("float16", 2, 128, [-1] * 16, [], cached, rows)
    batch = du.make_batch(plan)
    up = du.random_trees(np.random.default_rng(1), rows)
    q = du.queries(16 * 64, 16, 128, "float16")
    _, _, big, dev = run(plan, batch, q, du.offsets_of(rows), up)
    takes = parrot.load_library().parrot_test_tree_kernel
    assert takes(ctypes.byref(big.problem), ctypes.byref(big.rows), 0) == 0
    for n in (8, 3, 1):
        prob = problem_for(plan)
        prob.num_requests = n
        counts = parrot.make_tree_rows(64 * n, 64, 0, 16)
        assert takes(ctypes.byref(prob), ctypes.byref(counts), 0) == 2
        small = parrot.TreeDecoder(prob, counts)
        assert small.workspace.numel() <= big.workspace.numel()
        want, wlse = small(dev)
        big.workspace.fill_(0xFF)
        big.out.fill_(7.0)
        parrot.parrot_shared_prefix_tree_decode(
            prob, counts, dev["q_rows"], dev["query_offsets"], dev["tree_parents"], None, None, dev["k_pool"], dev["v_pool"],
            None, None, None, dev["suffix_tables"], dev["suffix_lens"], dev["group_ids"], big.out, big.lse, big.workspace)
        torch.cuda.synchronize()
        assert torch.equal(big.out[:64 * n], want) and torch.equal(big.lse[:64 * n], wlse)
        assert (big.out[64 * n:] == 7.0).all()
        part = [x[:64 * n] for x in (q, up)]
        few = du.tree_plan("float16", 2, 128, [-1] * n, [], cached[:n], rows[:n])
        few.suffix_tables, few.suffix_lens = plan.suffix_tables[:n], plan.suffix_lens[:n]
        if n == 1:
            check(few, batch, part[0], du.offsets_of(rows[:n]), part[1], want, wlse, what="one of sixteen")


def test_parents_that_stop_early(path):
    """Rows behind the end of the parents tensor are padding: left as they were, by tree
    decode and accept; requests before them are not touched by that."""
    import paper_2405_19888_amd as parrot
    plan, batch, off, up, q, rows, _ = batch_of("float16", 128, "32", seed=2)
    out, lse, dec, dev = run(plan, batch, q, off, up)
    want, n = out.clone(), int(off[2])
    held = dev["tree_parents"][:n].clone()
    dec.out.fill_(7.0)
    dec.bind({**dev, "tree_parents": held}, nested=True)()
    torch.cuda.synchronize()
    # (fewer rows may be cut otherwise: each result within the rounding of its weights)
    assert (dec.out[:n].double() - want[:n].double()).abs().max() <= 4 * du.UNIT["float16"] * 5
    assert (dec.out[n:] == 7.0).all()
    tokens = [torch.arange(off[-1], dtype=torch.int32).cuda() for _ in range(2)]
    ver = parrot.TreeVerifier(dec.problem, parrot.make_tree_rows(int(off[-1]), 16, 0, 4))
    ver.accept_rows.fill_(-77)
    ver.bind_accept({**dev, "tree_parents": held, "draft_tokens": tokens[0], "target_tokens": tokens[1],
                     "root_tokens": torch.zeros(3, dtype=torch.int32).cuda()})()
    torch.cuda.synchronize()
    assert (ver.accept_rows[n:] == -77).all() and (ver.accept_rows[:n] >= -1).all() and ver.accept_lens[2] == 0


@pytest.mark.parametrize("dtype,dim,most", [("float16", 128, 5), ("bfloat16", 64, 12), ("float32", 128, 9)])
def test_few_rows_with_prefixes(path, dtype, dim, most):
    """Two requests of seventy read long prefixes, in many chunks: the partial results of those
    rows alone are kept, and the others' stand elsewhere."""
    rng = np.random.default_rng(most)
    rows = [int(x) for x in rng.integers(0, most + 1, 70)]
    rows[9], rows[66] = most, most - 1
    cached = [int(x) for x in rng.integers(1, 60, 70)]
    groups = [-1] * 70
    groups[9], groups[66] = 1, 0
    plan = du.tree_plan(dtype, 2, dim, groups, [2900, 333], cached, rows, [-1, 0], seed=1)
    batch, off = du.make_batch(plan, seed=2), du.offsets_of(rows)
    up = du.random_trees(rng, rows)
    q = du.queries(int(off[-1]) + 4, 4, dim, dtype)
    out, lse, _, _ = run(plan, batch, q, off, up)
    check(plan, batch, q, off, up, out, lse, what=f"{path} {dtype} {dim} few rows with prefixes")
