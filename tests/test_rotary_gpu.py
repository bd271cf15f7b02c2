"""GPU parity of the fill of new rows: layouts, part of the head, scalings, far
positions, norms, strides, padding, and what stays untouched."""
import math

import numpy as np
import pytest
import torch

import drafts_util as du
from drafts_util import oracle

pytestmark = pytest.mark.gpu

EPS = 1e-6


def tolerance(dtype, y, size, weight):
    """One rounding to the type, and the fp32 errors: sine and cosine (3.5 steps of 2^-24
    from the angle's conversion and the series), the products with weight and amplitude,
    the sum, and with a norm the sum of squares (13 steps, halved by the root), root,
    division and scaling: 20 steps of 2^-24 of the pair's size in all."""
    w = 1.0 if weight is None else float(np.abs(weight).max())
    return du.UNIT[dtype] * np.abs(y) * 1.01 + 20 * du.F32 * size * max(1.0, w) + 1e-30


def rows_of(seed, T, heads, dim, dtype, scale=1.0):
    return du.queries(T, heads, dim, dtype, seed=seed) * scale


def setup(dtype, heads, dim, cached, rows, seed=0):
    plan = du.tree_plan(dtype, heads, dim, [-1] * len(rows), [], cached, rows, seed=seed)
    return plan, du.make_batch(plan, seed=seed), du.offsets_of(rows)


def fill(plan, batch, off, q, k, v, positions, rotary, T=None, q_norm=None, k_norm=None, eps=EPS, fused=True):
    import paper_2405_19888_amd as parrot
    dev = batch.to("cuda")
    T = k.shape[0] if T is None else T
    if fused:                        # slices of one projection's output
        x = torch.cat([y.flatten(1) for y in (q, k, v)], 1).cuda()
        parts = x.split([y[0].numel() for y in (q, k, v)], 1)
        dev["q_rows"], dev["k_rows"], dev["v_rows"] = (p.unflatten(1, y.shape[1:]) for p, y in zip(parts, (q, k, v)))
    else:
        dev["q_rows"], dev["k_rows"], dev["v_rows"] = q.cuda(), k.cuda(), v.cuda()
    dev["positions"] = torch.tensor(positions, dtype=torch.int32).cuda()
    dev["query_offsets"] = torch.from_numpy(off).cuda()
    dev["q_norm"] = None if q_norm is None else q_norm.cuda()
    dev["k_norm"] = None if k_norm is None else k_norm.cuda()
    prob = parrot.make_problem(
        num_requests=len(off) - 1, num_heads=plan.heads, head_dim=plan.head_dim, block_size=16, num_groups=0,
        max_group_size=0, max_prefix_len=0, max_suffix_len=int(plan.suffix_lens.max()), prefix_table_stride=0,
        suffix_table_stride=plan.suffix_tables.shape[1], num_prefix_blocks=0, num_suffix_blocks=plan.num_blocks,
        dtype=du.TORCH_DTYPES[plan.dtype], sm_scale=1.0)
    f = parrot.RotaryFiller(prob, T, int(np.diff(off).max()), q.shape[1], rotary=rotary, norm_eps=eps)
    f.q_out.fill_(float("nan"))
    f(dev)
    torch.cuda.synchronize()
    return f, dev


def check(plan, batch, off, q, k, v, positions, radians, amplitude, interleaved, f, dev, q_norm=None, k_norm=None,
          what=""):
    n = int(off[-1])
    assert torch.isnan(f.q_out[n:]).all(), "padding rows were written"
    want, size = oracle.rotate(q[:n], positions[:n], radians, interleaved, amplitude, q_norm, EPS)
    err = np.abs(f.q_out[:n].double().cpu().numpy() - want)
    worst = (err / tolerance(plan.dtype, want, size, None if q_norm is None else q_norm.double().numpy())).max()
    kw, ks = oracle.rotate(k[:n], positions[:n], radians, interleaved, amplitude, k_norm, EPS)
    ktol = tolerance(plan.dtype, kw, ks, None if k_norm is None else k_norm.double().numpy())
    kp, vp = dev["k_pool"].cpu(), dev["v_pool"].cpu()
    before_k, before_v = batch.k_pool.clone(), batch.v_pool.clone()
    kworst = 0.0
    for row, blk, at in oracle.fill_slots(off, plan.suffix_tables, plan.suffix_lens):
        kworst = max(kworst, (np.abs(kp[blk, :, at].double().numpy() - kw[row]) / ktol[row]).max())
        assert torch.equal(vp[blk, :, at], v[row]), "values are copied"
        before_k[blk, :, at], before_v[blk, :, at] = kp[blk, :, at], vp[blk, :, at]
    same = lambda a, b: torch.equal(torch.nan_to_num(a, 123.0), torch.nan_to_num(b, 123.0))
    assert same(before_k, kp) and same(before_v, vp), "another slot was written"
    print(f"{what}: q {worst:.2f}, k {kworst:.2f} of the bound", flush=True)
    assert worst <= 1.0 and kworst <= 1.0, (what, worst, kworst)


@pytest.mark.parametrize("dtype,dim", [("float16", 128), ("bfloat16", 128), ("float32", 128), ("float16", 64),
                                       ("float32", 64)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rd", ["whole", "half", 2, 20, 50])
def test_layouts(dtype, dim, interleaved, rd):
    """Whole heads, half of them, and odd parts that no 16 bytes line up with."""
    import paper_2405_19888_amd as parrot
    rd = {"whole": dim, "half": dim // 2}.get(rd, rd)
    cached, rows = [0, 15, 100, 31], [3, 1, 18, 2]
    plan, batch, off = setup(dtype, 3, dim, cached, rows)
    T = int(off[-1]) + 2
    q, k, v = rows_of(1, T, 6, dim, dtype), rows_of(2, T, 3, dim, dtype), rows_of(3, T, 3, dim, dtype)
    positions = list(np.random.default_rng(rd).integers(0, 5000, T))
    rotary = parrot.make_rotary(rd, interleaved=interleaved)
    radians, amplitude = oracle.rotary_frequencies(rd)
    for norm in (False, True):
        qn, kn = (1 + 0.2 * rows_of(4, 2, 1, dim, dtype)[:, 0]).unbind(0) if norm else (None, None)
        f, dev = fill(plan, batch, off, q, k, v, positions, rotary, q_norm=qn, k_norm=kn, fused=not norm)
        check(plan, batch, off, q, k, v, positions, radians, amplitude, interleaved, f, dev, qn, kn,
              f"{dtype} {dim} rd {rd} interleaved {interleaved} norm {norm}")


@pytest.mark.parametrize("scaling,factor", [("linear", 4.0), ("ntk", 8.0), ("yarn", 16.0), ("wavelength", 8.0)])
def test_scalings_and_far_positions(scaling, factor):
    """Angles hold at positions up to 2^31 - 1, and below 0."""
    import paper_2405_19888_amd as parrot
    plan, batch, off = setup("float32", 2, 128, [10, 3], [6, 5])
    q, k, v = rows_of(1, 11, 2, 128, "float32"), rows_of(2, 11, 2, 128, "float32"), rows_of(3, 11, 2, 128, "float32")
    positions = [0, 1, 4096, 131071, 1 << 20, (1 << 24) + 1, 10 ** 7 + 3, 2 ** 29 + 5, 2 ** 31 - 1, -1, -99999]
    rotary = parrot.make_rotary(128, base=500000.0, scaling=scaling, factor=factor, original_length=4096)
    radians, amplitude = oracle.rotary_frequencies(128, 500000.0, scaling, factor, 4096)
    f, dev = fill(plan, batch, off, q, k, v, positions, rotary)
    # the 64-bit angle itself is exact to 2^31 * 2^-53 = 2.4e-7 radians at the far end:
    # four more steps of 2^-24
    err = np.abs(f.q_out.double().cpu().numpy() - oracle.rotate(q, positions, radians, False, amplitude)[0])
    bound = 24 * du.F32 * oracle.rotate(q, positions, radians, False, amplitude)[1] + du.F32
    assert (err <= bound).all(), (err / bound).max()


@pytest.mark.parametrize("dtype", ["float16", "float32"])
def test_norm_only_keys_only_in_place(dtype):
    import paper_2405_19888_amd as parrot
    plan, batch, off = setup(dtype, 2, 64, [5, 40], [7, 2])
    q, k, v = rows_of(1, 9, 4, 64, dtype), rows_of(2, 9, 2, 64, dtype), rows_of(3, 9, 2, 64, dtype)
    w = 1 + 0.1 * rows_of(9, 1, 1, 64, dtype)[0, 0]
    f, dev = fill(plan, batch, off, q, k, v, [0] * 9, None, q_norm=None, k_norm=w)
    check(plan, batch, off, q, k, v, [0] * 9, [], 1.0, False, f, dev, None, w, "keys normed, queries copied")
    assert torch.equal(f.q_out.cpu(), q)
    f, dev = fill(plan, batch, off, q, k, v, [0] * 9, None, q_norm=w, k_norm=None)
    check(plan, batch, off, q, k, v, [0] * 9, [], 1.0, False, f, dev, w, None, "queries normed")
    # keys and values only
    fresh = batch.to("cuda")
    t = dict(dev, k_pool=fresh["k_pool"], v_pool=fresh["v_pool"])
    only = parrot.RotaryFiller(f.problem, 9, 7, 0)
    assert only(t) is None
    torch.cuda.synchronize()
    same = lambda a, b: torch.equal(torch.nan_to_num(a, 123.0), torch.nan_to_num(b, 123.0))
    assert same(fresh["k_pool"], dev["k_pool"]) and same(fresh["v_pool"], dev["v_pool"])
    # in place, rotated
    rot = parrot.make_rotary(64)
    want, _ = fill(plan, batch, off, q, k, v, list(range(9)), rot, fused=False)
    x = q.cuda()
    parrot.parrot_rotary_fill(f.problem, 9, 7, 4, rot, x, k.cuda(), v.cuda(), None, None,
                              torch.arange(9, dtype=torch.int32).cuda(), torch.from_numpy(off).cuda(),
                              dev["suffix_tables"], dev["suffix_lens"], x, dev["k_pool"], dev["v_pool"])
    torch.cuda.synchronize()
    assert torch.equal(x, want.q_out)


def test_infinite_and_nan_elements_stay_in_their_pair():
    import paper_2405_19888_amd as parrot
    plan, batch, off = setup("float16", 1, 64, [3], [2])
    q, k, v = rows_of(1, 2, 1, 64, "float16"), rows_of(2, 2, 1, 64, "float16"), rows_of(3, 2, 1, 64, "float16")
    for rd, interleaved, partner in ((32, False, 21), (32, True, 4), (20, False, 15)):
        rot = parrot.make_rotary(rd, interleaved=interleaved)
        clean, _ = fill(plan, batch, off, q, k, v, [7, 8], rot)
        clean = clean.q_out.clone()
        x = q.clone()
        x[0, 0, 5] = float("inf")
        x[1, 0, rd] = float("nan")                        # outside the rotated part
        got, _ = fill(plan, batch, off, x, k, v, [7, 8], rot)
        got = got.q_out
        other = [i for i in range(64) if i not in (5, partner)]
        assert torch.equal(got[0, 0, other], clean[0, 0, other])
        other = [i for i in range(64) if i != rd]
        assert torch.equal(got[1, 0, other], clean[1, 0, other]) and torch.isnan(got[1, 0, rd])


def test_many_rows_and_requests():
    """More rows than workgroup slots, more requests than a wave, empty requests."""
    import paper_2405_19888_amd as parrot
    rng = np.random.default_rng(5)
    rows = [int(x) for x in rng.integers(0, 9, 300)]
    cached = [int(x) for x in rng.integers(1, 40, 300)]
    plan, batch, off = setup("bfloat16", 2, 128, cached, rows, seed=2)
    T = int(off[-1])
    q, k, v = rows_of(1, T, 10, 128, "bfloat16"), rows_of(2, T, 2, 128, "bfloat16"), rows_of(3, T, 2, 128, "bfloat16")
    positions = list(rng.integers(0, 9000, T))
    f, dev = fill(plan, batch, off, q, k, v, positions, parrot.make_rotary(128))
    radians, amplitude = oracle.rotary_frequencies(128)
    check(plan, batch, off, q, k, v, positions, radians, amplitude, False, f, dev, what="300 requests")


def test_graph_and_one_call_form():
    import paper_2405_19888_amd as parrot
    plan, batch, off = setup("float16", 2, 128, [9, 30], [4, 3])
    q, k, v = rows_of(1, 7, 2, 128, "float16"), rows_of(2, 7, 2, 128, "float16"), rows_of(3, 7, 2, 128, "float16")
    rot = parrot.make_rotary(128)
    f, dev = fill(plan, batch, off, q, k, v, list(range(7)), rot)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(dev)
    for i in range(3):
        dev["positions"].add_(11 * (i + 1))
        f.q_out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got, gk = f.q_out.clone(), dev["k_pool"].clone()
        out = parrot.rotary_fill(dev["q_rows"], dev["k_rows"], dev["v_rows"], dev["positions"], dev["query_offsets"],
                                 dev["k_pool"], dev["v_pool"], dev["suffix_tables"], dev["suffix_lens"], rotary=rot)
        torch.cuda.synchronize()
        assert torch.equal(out, got) and torch.equal(torch.nan_to_num(gk), torch.nan_to_num(dev["k_pool"]))


@pytest.mark.parametrize("dtype,dim,interleaved,rd", [("float16", 128, False, 128), ("bfloat16", 128, False, 96),
                                                      ("float32", 128, False, 20), ("float16", 64, True, 64),
                                                      ("bfloat16", 64, False, 12)])
@pytest.mark.parametrize("requests", [2, 300])
def test_in_place_over_many_heads(dtype, dim, interleaved, rd, requests):
    """Queries rotated in place, several steps of a row's heads requested ahead, by few rows
    (a row's heads over several workgroups) and by many."""
    import paper_2405_19888_amd as parrot
    rows = [5] * requests
    plan, batch, off = setup(dtype, 8, dim, [3] * requests, rows)
    T = 5 * requests
    q, k, v = (rows_of(i, T, h, dim, dtype) for i, h in ((1, 72), (2, 8), (3, 8)))
    w = 1 + 0.1 * rows_of(9, 1, 1, dim, dtype)[0, 0]
    rot = parrot.make_rotary(rd, interleaved=interleaved)
    positions = [int(x) for x in np.random.default_rng(0).integers(0, 9000, T)]
    want, dev = fill(plan, batch, off, q, k, v, positions, rot, q_norm=w, k_norm=w)
    x = q.cuda()
    parrot.parrot_rotary_fill(want.problem, T, 5, 72, rot, x, k.cuda(), v.cuda(), dev["q_norm"], dev["k_norm"],
                              dev["positions"], dev["query_offsets"], dev["suffix_tables"], dev["suffix_lens"], x,
                              dev["k_pool"], dev["v_pool"], norm_eps=EPS)
    torch.cuda.synchronize()
    assert torch.equal(x, want.q_out)
