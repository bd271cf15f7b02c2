"""GPU parity of attention for drafted trees: types, head layouts, tree shapes, ragged
and odd lengths, nested and flat prefixes, padding, what masked tokens hold."""
import numpy as np
import pytest
import torch

import drafts_util as du
from drafts_util import oracle
from gpu_util import problem_for

pytestmark = pytest.mark.gpu

PATHS = {"one": 0, "split": 1}


@pytest.fixture(autouse=True, params=["one", "split"])
def path(request):
    """Every test runs on one launch, and on partial results and join."""
    import paper_2405_19888_amd as parrot
    force = parrot.load_library().parrot_test_tree_path
    force(PATHS[request.param])
    yield request.param
    force(-1)


def run(plan, batch, q, off, parents, T=None, trees=True):
    """One call on poisoned outputs; (out, lse, decoder, device tensors)."""
    import paper_2405_19888_amd as parrot
    dev = batch.to("cuda")
    dev["q_rows"], dev["query_offsets"] = q.cuda(), torch.from_numpy(off).cuda()
    dev["tree_parents"] = torch.from_numpy(parents).cuda() if trees else None
    rows = parrot.tree_rows_from_host(off, plan.group_ids, plan.num_groups, q.shape[1],
                                      plan.prefix_parents if plan.nested else None)
    rows.num_query_rows = q.shape[0] if T is None else T
    prob = problem_for(plan)
    scratch = torch.zeros(16, dtype=torch.int32, device="cuda")
    parrot.parrot_validate_tree_inputs(prob, rows, dev["query_offsets"], dev["tree_parents"], dev["prefix_tables"],
                                       dev["prefix_lens"], dev["prefix_parents"] if plan.nested else None,
                                       dev["suffix_tables"], dev["suffix_lens"], dev["group_ids"], scratch)
    dec = parrot.TreeDecoder(prob, rows)
    dec.out.fill_(float("nan"))
    dec.lse.fill_(float("nan"))
    dec.workspace.fill_(0xFF)
    dec(dev, nested=plan.nested)
    torch.cuda.synchronize()
    return dec.out, dec.lse, dec, dev


def check(plan, batch, q, off, parents, out, lse, trees=True, what=""):
    kp, vp = batch.k_pool, batch.v_pool
    ref, rlse, spread, noise = oracle.shared_prefix_tree(
        q, off, parents if trees else None, kp, vp, kp, vp, plan.prefix_tables, plan.prefix_lens, plan.suffix_tables,
        plan.suffix_lens, plan.group_ids, plan.sm_scale, plan.prefix_parents if plan.nested else None)
    n = int(off[-1])
    keys = int(plan.suffix_lens.max()) + int(plan.prefix_lens.sum() if plan.nested else max([0] + list(plan.prefix_lens)))
    got, glse = out.double().cpu().numpy()[:n], lse.double().cpu().numpy()[:n]
    tol = du.out_tolerance(plan.dtype, ref[:n], spread[:n], noise[:n], keys, plan.head_dim)
    ltol = du.lse_tolerance(rlse[:n], noise[:n], keys, plan.head_dim)
    assert np.isfinite(got).all() and np.isfinite(glse).all(), what
    worst = (np.abs(got - ref[:n]) / tol).max()
    lworst = (np.abs(glse - rlse[:n]) / ltol).max()
    print(f"{what}: out error {worst:.2f} of its bound, lse {lworst:.2f}", flush=True)
    assert worst <= 1.0 and lworst <= 1.0, (what, worst, lworst)
    assert torch.isnan(out[n:]).all() and torch.isnan(lse[n:]).all(), "padding rows were written"


# (dtype, heads, ratio, dim, group of request, prefix lengths, cached, rows, parents)
CASES = {
    "f32_small": ("float32", 4, 1, 64, [0, 0, 0, 0], [128], [16, 24, 32, 20], [4, 4, 4, 4], None),
    "one_row_no_cache": ("float16", 2, 1, 128, [-1], [], [0], [1], None),
    "one_row_each": ("bfloat16", 3, 4, 128, [-1, 0, -1], [33], [1, 0, 15], [1, 1, 1], None),
    "tree_only": ("float16", 2, 2, 64, [-1, -1], [], [0, 0], [128, 17], None),
    "odd_lengths": ("bfloat16", 5, 1, 128, [0, -1, 1, 0, 1], [1, 47], [31, 32, 33, 0, 100], [1, 2, 33, 64, 15], None),
    "base_alignments": ("float16", 1, 8, 64, [-1] * 8, [], [27, 28, 29, 30, 31, 32, 63, 65], [5, 6, 7, 8, 33, 1, 2, 70], None),
    "many_columns": ("float16", 2, 8, 128, [-1, 0], [40], [50, 300], [40, 128], None),
    "ratio_seven_f32": ("float32", 2, 7, 128, [0, -1, 0], [75], [3, 90, 17], [19, 9, 30], None),
    "nested": ("bfloat16", 4, 2, 128, [1, 2, 0, 3, -1, 3], [70, 16, 5, 130], [12, 0, 7, 40, 64, 1],
               [8, 3, 5, 1, 12, 20], [-1, 0, 0, 1]),
    "long_own": ("float16", 2, 4, 128, [-1, 0], [2100], [4700, 2049], [13, 30], None),
    "no_rows_between": ("float16", 4, 1, 64, [0, 0, -1, 0], [64], [9, 10, 11, 12], [0, 3, 0, 2], None),
    "f32_long": ("float32", 2, 1, 64, [0], [600], [2500], [40], None),
    "f32_two_sets": ("float32", 3, 1, 128, [0, -1, 0], [40], [70, 200, 0], [20, 32, 17], None),
    # few runs of a head, two tiles beside single ones: the tiles are cut at the same tokens
    "cut_together": ("float16", 40, 8, 128, [-1, -1, -1, -1], [], [1480, 1500, 900, 300], [20, 5, 3, 9], None),
    # more tiles that share keys than a quarter of the runs: cut where they fall
    "cut_apart": ("bfloat16", 40, 8, 64, [0, -1, -1, 0], [100], [500, 700, 30, 0], [20, 33, 40, 50], None),
    # prefix chunks longer than the runs of own tokens, and shorter
    "prefix_first": ("float16", 2, 2, 128, [0, 0, 1, 1, -1], [900, 257], [20, 0, 31, 64, 3], [40, 33, 3, 40, 20], None),
    "own_first": ("bfloat16", 1, 1, 64, [0, -1], [80], [9000, 700], [30, 31], None),
    "heads_odd": ("float16", 7, 3, 128, [0, 1, -1], [15, 333], [130, 65, 2], [11, 22, 33], [-1, 0]),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("trees", [True, False])
def test_tree_parity(name, trees):
    dtype, heads, ratio, dim, groups, plen, cached, rows, parents = CASES[name]
    rng = np.random.default_rng(len(name))
    plan = du.tree_plan(dtype, heads, dim, groups, plen, cached, rows, parents, seed=3)
    batch, off = du.make_batch(plan, seed=5), du.offsets_of(rows)
    up = du.random_trees(rng, rows, spread=int(rng.integers(1, 9)), roots=int(rng.integers(1, 3)))
    q = du.queries(int(off[-1]) + 3, heads * ratio, dim, dtype)          # three rows of padding
    out, lse, _, _ = run(plan, batch, q, off, up, trees=trees)
    check(plan, batch, q, off, up, out, lse, trees=trees, what=name)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.5])
def test_scales(scale):
    """Negative, zero and large scales (logits up to about 60)."""
    for dtype in ("float16", "float32"):
        plan = du.tree_plan(dtype, 2, 64, [0, -1], [50], [20, 70], [6, 9], scale=scale)
        batch, off = du.make_batch(plan), du.offsets_of([6, 9])
        up = du.random_trees(np.random.default_rng(1), [6, 9])
        q = du.queries(15, 4, 64, dtype)
        out, lse, _, _ = run(plan, batch, q, off, up)
        check(plan, batch, q, off, up, out, lse, what=f"{dtype} scale {scale}")


@pytest.mark.parametrize("dtype,dim", [("float16", 128), ("bfloat16", 64), ("float32", 128), ("float32", 64)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_masked_tokens_hold_anything(dtype, dim, value):
    """A drafted token's K and V reach only the rows that see it: with its value (and
    key) not finite, every other row's result is bit for bit the one of finite values,
    and the rows that see the value get it where it stands."""
    rows, cached = [20, 9], [37, 3]
    plan = du.tree_plan(dtype, 2, dim, [0, -1], [18], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    up = du.random_trees(np.random.default_rng(2), rows)
    q = du.queries(29, 4, dim, dtype)
    clean, clse, _, dev = run(plan, batch, q, off, up)
    token, d = 11, 5                                           # drafted row 11 of request 0, one element of head 1
    pos = cached[0] + token
    blk = int(plan.suffix_tables[0][pos // 16])
    sees = np.array([token in oracle.tree_path(up[:20], j) for j in range(20)] + [False] * 9)
    batch.v_pool[blk, 1, pos % 16, d] = value
    got, glse, _, _ = run(plan, batch, q, off, up)
    assert torch.equal(got[~sees], clean[~sees]) and torch.equal(glse, clse)
    hit = got[sees][:, 2:]                                     # query heads 2, 3 read cache head 1
    assert torch.equal(torch.isnan(hit[..., d]), torch.isnan(torch.full_like(hit[..., d], value)))
    if value == value:
        assert torch.equal(hit[..., d], torch.full_like(hit[..., d], value))
    rest = [i for i in range(dim) if i != d]
    assert torch.equal(hit[..., rest], clean[sees][:, 2:][..., rest])
    batch.k_pool[blk, 1, pos % 16, :] = value
    got, _, _, _ = run(plan, batch, q, off, up)
    assert torch.equal(got[~sees], clean[~sees])
    assert torch.isnan(got[sees][:, 2:][..., d]).all()


def test_bad_parents_stay_in_bounds():
    """Parents that break the rules are refused by the check, and a call that skipped it
    treats them as -1."""
    import paper_2405_19888_amd as parrot
    rows, cached = [7, 5], [20, 40]
    plan = du.tree_plan("float16", 2, 64, [-1, -1], [], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    up = np.array([-1, 0, 1, 1, 3, 2, 0, -1, 0, 1, 2, 2], np.int32)
    q = du.queries(12, 2, 64, "float16")
    good, _, dec, dev = run(plan, batch, q, off, up)
    good = good.clone()
    bad = up.copy()
    bad[0], bad[7] = 1 << 30, -5
    dev["tree_parents"] = torch.from_numpy(bad).cuda()
    scratch = torch.zeros(16, dtype=torch.int32, device="cuda")
    with pytest.raises(parrot.ParrotError, match="tree parent"):
        parrot.parrot_validate_tree_inputs(dec.problem, dec.rows, dev["query_offsets"], dev["tree_parents"],
                                           dev["prefix_tables"], dev["prefix_lens"], None, dev["suffix_tables"],
                                           dev["suffix_lens"], dev["group_ids"], scratch)
    dec(dev)
    torch.cuda.synchronize()
    assert torch.equal(dec.out, good)


def test_chain_equals_prefill():
    """A chain with one query head per cache head is the prefill of those rows."""
    from gpu_util import run_prefill
    rows, cached = [16, 5, 30], [100, 3, 64]
    plan = du.tree_plan("float16", 4, 128, [0, 0, -1], [200], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    q = du.queries(51, 4, 128, "float16")
    out, lse, _, dev = run(plan, batch, q, off, np.zeros(51, np.int32), trees=False)
    pout, plse = run_prefill(plan, dev, off)
    # both are within the rounding of their weights: 2 units of 16 bits of values up to 5
    assert (out.double() - pout.double()).abs().max() <= 4 * du.UNIT["float16"] * 5
    assert (lse - plse).abs().max() <= 1e-4


def test_other_stream_and_graph():
    """The call on a stream of its own, and captured: replays follow the inputs, with
    eager work between them, and fewer rows than the graph was captured with."""
    import paper_2405_19888_amd as parrot
    rows, cached = [6, 11], [50, 300]
    plan = du.tree_plan("bfloat16", 2, 128, [0, -1], [90], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    rng = np.random.default_rng(0)
    up = du.random_trees(rng, rows)
    q = du.queries(17, 8, 128, "bfloat16")
    out, lse, dec, dev = run(plan, batch, q, off, up)
    want, wlse = out.clone(), lse.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    dec.out.zero_()
    torch.cuda.synchronize()
    dec(dev, stream=s)
    s.synchronize()
    assert torch.equal(dec.out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dec(dev)
    for i in range(3):
        dec.out.fill_(float("nan"))
        dev["q_rows"].copy_(du.queries(17, 8, 128, "bfloat16", seed=i))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = dec.out.clone()
        dec(dev)
        torch.cuda.synchronize()
        assert torch.equal(got, dec.out), f"replay {i}"
    # the second request brings 4 rows now, the rest is padding
    dev["query_offsets"].copy_(torch.tensor([0, 6, 10]))
    dev["suffix_lens"][1] -= 7
    dec.out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert (dec.out[10:] == 7.0).all() and torch.isfinite(dec.out[:10].float()).all()


def test_one_call_form():
    import paper_2405_19888_amd as parrot
    rows, cached = [5, 8], [10, 20]
    plan = du.tree_plan("float16", 2, 64, [0, 0], [33], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    up = du.random_trees(np.random.default_rng(4), rows)
    q = du.queries(13, 6, 64, "float16")
    want, wlse, _, dev = run(plan, batch, q, off, up)
    out, lse = parrot.tree_decode(dev["q_rows"], dev["query_offsets"], dev["tree_parents"], dev["k_pool"],
                                  dev["v_pool"], dev["k_pool"], dev["v_pool"], dev["prefix_tables"],
                                  dev["prefix_lens"], dev["suffix_tables"], dev["suffix_lens"], dev["group_ids"])
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    # on another stream, the allocator busy on this one
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got, _ = parrot.tree_decode(dev["q_rows"], dev["query_offsets"], dev["tree_parents"], dev["k_pool"],
                                    dev["v_pool"], dev["k_pool"], dev["v_pool"], dev["prefix_tables"],
                                    dev["prefix_lens"], dev["suffix_tables"], dev["suffix_lens"], dev["group_ids"], stream=s)
        torch.full((1 << 16,), 0xFF, dtype=torch.uint8, device="cuda")
        s.synchronize()
        assert torch.equal(got, want)


def test_seeded_random_plans():
    rng = np.random.default_rng(11)
    for i in range(12):
        dtype = ["float16", "bfloat16", "float32"][i % 3]
        heads, ratio = [(1, 8), (4, 1), (2, 3), (3, 5)][int(rng.integers(4))]
        dim = [64, 128][int(rng.integers(2))]
        R, ng = int(rng.integers(1, 7)), int(rng.integers(0, 4))
        plen = [int(x) for x in rng.integers(1, 400, ng)]
        parents = [-1] + [int(rng.integers(-1, g)) for g in range(1, ng)] if ng and i % 2 else None
        groups = [int(x) for x in rng.integers(-1, ng, R)] if ng else [-1] * R
        rows = [int(x) for x in rng.integers(0, 41, R)]
        rows[0] = max(rows[0], 1)
        cached = [int(x) for x in rng.integers(0, 700, R)]
        if any(c + n == 0 and g < 0 for c, n, g in zip(cached, rows, groups)):
            cached = [c + 1 for c in cached]
        plan = du.tree_plan(dtype, heads, dim, groups, plen, cached, rows, parents, seed=i)
        batch, off = du.make_batch(plan, seed=i), du.offsets_of(rows)
        up = du.random_trees(rng, rows, spread=int(rng.integers(1, 12)))
        q = du.queries(int(off[-1]) + 1, heads * ratio, dim, dtype, seed=i)
        out, lse, _, _ = run(plan, batch, q, off, up)
        check(plan, batch, q, off, up, out, lse, what=f"plan {i} {dtype} {heads}x{ratio}x{dim}")


@pytest.mark.parametrize("dtype,dim,most", [("float16", 128, 3), ("float32", 64, 3), ("bfloat16", 64, 30)])
def test_more_requests_than_threads(dtype, dim, most):
    """300 requests: lengths and rows are summed in two passes, some bring no rows."""
    rng = np.random.default_rng(8)
    rows = [int(x) for x in rng.integers(0, most + 1, 300)]
    cached = [int(x) for x in rng.integers(0, 90, 300)]
    groups = [int(x) for x in rng.integers(-1, 3, 300)]
    cached = [c + 1 if c + n == 0 and g < 0 else c for c, n, g in zip(cached, rows, groups)]
    plan = du.tree_plan(dtype, 2, dim, groups, [50, 7, 140], cached, rows, [-1, 0, -1])
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    up = du.random_trees(rng, rows)
    q = du.queries(int(off[-1]), 4, dim, dtype)
    out, lse, _, _ = run(plan, batch, q, off, up)
    check(plan, batch, q, off, up, out, lse, what=f"300 requests {dtype}")


def test_two_calls_at_once():
    """Two handles on two streams, over the same caches."""
    import paper_2405_19888_amd as parrot
    rows, cached = [12, 40, 5], [900, 2000, 64]
    plan = du.tree_plan("bfloat16", 4, 128, [0, -1, 0], [700], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    up = du.random_trees(np.random.default_rng(3), rows)
    q = du.queries(57, 8, 128, "bfloat16")
    want, wlse, first, dev = run(plan, batch, q, off, up)
    want = want.clone()
    second = parrot.TreeDecoder(first.problem, first.rows)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for dec, s in zip((first, second), streams):
            dec(dev, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(first.out, want) and torch.equal(second.out, want)


def test_two_graphs_of_one_handle():
    """Graphs of one handle share its workspace; replayed one after the other, with eager
    calls between them, each gives its own inputs' result."""
    import paper_2405_19888_amd as parrot
    rows, cached = [9, 21], [500, 300]
    plan = du.tree_plan("float16", 2, 128, [0, 0], [260], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    up = du.random_trees(np.random.default_rng(3), rows)
    qs = [du.queries(30, 8, 128, "float16", seed=i) for i in range(2)]
    _, _, dec, dev = run(plan, batch, qs[0], off, up)
    devs, graphs, want = [], [], []
    for x in qs:
        devs.append({**dev, "q_rows": x.cuda()})
        dec(devs[-1])
        torch.cuda.synchronize()
        want.append(dec.out.clone())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            dec(devs[-1])
    for i in (0, 1, 1, 0, 1):
        dec(devs[1 - i])
        torch.cuda.synchronize()
        dec.out.fill_(float("nan"))
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(dec.out, want[i])


def test_flat_call_with_a_nested_problem():
    """A flat call of a problem that allows nested groups uses the same workspace."""
    import paper_2405_19888_amd as parrot
    rows, cached = [10, 20, 7], [100, 30, 64]
    plan = du.tree_plan("float16", 2, 128, [0, 1, -1], [300, 90], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    up = du.random_trees(np.random.default_rng(5), rows)
    q = du.queries(37, 4, 128, "float16")
    want, _, dec, dev = run(plan, batch, q, off, up)
    want = want.clone()
    prob = problem_for(plan)
    prob.max_prefix_depth = 4
    deep = parrot.TreeDecoder(prob, dec.rows)
    deep.workspace.fill_(0xFF)
    deep(dev, nested=False)
    torch.cuda.synchronize()
    # the same keys in other pieces: each within the rounding of its weights
    assert (deep.out.double() - want.double()).abs().max() <= 4 * du.UNIT["float16"] * 5
