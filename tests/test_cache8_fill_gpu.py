"""GPU parity of the fill of a cache held in 8 bits: codes, scales, kept tokens, rotations and
norms, block edges, padding, strides, and what stays untouched."""
import numpy as np
import pytest
import torch

import cache8_util as cu
from cache8_util import du, drafts_oracle, oracle

pytestmark = pytest.mark.gpu

EPS = 1e-6
# errors of a key before its code, in steps of 2^-24 of its pair's size (see the 16-bit fill's test)
STEPS = 20


def setup(dtype, heads, dim, cached, rows, seed=0):
    plan = du.tree_plan(dtype, heads, dim, [-1] * len(rows), [], cached, rows, seed=seed)
    return plan, du.make_batch(plan, seed=seed), du.offsets_of(rows)


def random_pool(plan, seed, small=1.0):
    """Codes and scales of a whole pool, token order."""
    rng = np.random.default_rng(seed)
    n, h, d = plan.num_blocks, plan.heads, plan.head_dim
    out = []
    for _ in range(2):
        x = rng.normal(size=(n, h, 16, d)) * small * 2.0 ** rng.integers(-3, 4, (n, h, 1, 1))
        out.append(oracle.pack(x))
    return out


def fill(plan, off, pool, q, k, v, positions=None, rotary=None, T=None, q_norm=None, k_norm=None, fused=True, max_rows=None):
    import paper_2405_19888_amd as parrot
    T = k.shape[0] if T is None else T
    t = {}
    if fused:                        # slices of one projection's output
        parts = [y for y in (q, k, v) if y is not None]
        x = torch.cat([y.flatten(1) for y in parts], 1).cuda()
        split = [p.unflatten(1, y.shape[1:]) for p, y in zip(x.split([y[0].numel() for y in parts], 1), parts)]
        t["q_rows"] = split[0] if q is not None else None
        t["k_rows"], t["v_rows"] = split[-2:]
    else:
        t["q_rows"], t["k_rows"], t["v_rows"] = None if q is None else q.cuda(), k.cuda(), v.cuda()
    t["positions"] = None if positions is None else torch.tensor(positions, dtype=torch.int32).cuda()
    t["query_offsets"] = torch.from_numpy(off).cuda()
    t["suffix_tables"], t["suffix_lens"] = torch.from_numpy(plan.suffix_tables).cuda(), torch.from_numpy(plan.suffix_lens).cuda()
    t["q_norm"] = None if q_norm is None else q_norm.cuda()
    t["k_norm"] = None if k_norm is None else k_norm.cuda()
    (ck, bk), (cv, bv) = pool
    t["suffix"] = cu.device_pools(ck, oracle.value_order(cv), np.stack([bk, bv], -1))
    prob = parrot.make_problem(
        num_requests=len(off) - 1, num_heads=plan.heads, head_dim=plan.head_dim, block_size=16, num_groups=0,
        max_group_size=0, max_prefix_len=0, max_suffix_len=int(plan.suffix_lens.max()), prefix_table_stride=0,
        suffix_table_stride=plan.suffix_tables.shape[1], num_prefix_blocks=0, num_suffix_blocks=plan.num_blocks,
        dtype=du.TORCH_DTYPES[plan.dtype], sm_scale=1.0)
    f = parrot.Cache8Filler(prob, T, int(np.diff(off).max()) if max_rows is None else max_rows,
                            0 if q is None else q.shape[1], rotary=rotary, norm_eps=EPS)
    if q is not None:
        f.q_out.fill_(float("nan"))
    f(t)
    torch.cuda.synchronize()
    got = [(t["suffix"]["k"].view(torch.uint8).cpu().numpy(), t["suffix"]["scales"].view(torch.uint8)[..., 0].cpu().numpy()),
           (oracle.token_order(t["suffix"]["v"].view(torch.uint8).cpu().numpy()),
            t["suffix"]["scales"].view(torch.uint8)[..., 1].cpu().numpy())]
    return f, got, t


def same(got, want, what):
    assert np.array_equal(got[1], want[1]), f"{what}: scales"
    a, b = got[0], want[0]
    zero = (a % 128 == 0) & (b % 128 == 0)
    assert np.array_equal(np.where(zero, 0, a), np.where(zero, 0, b)), f"{what}: codes"


CASES = {
    # (dtype, heads, ratio, dim, cached, rows)
    "one": ("float16", 1, 1, 128, [0], [1]),
    "tokens": ("float16", 4, 2, 128, [0, 1, 3, 4, 15, 16, 17, 40], [1] * 8),
    "tokens_bf16_64": ("bfloat16", 3, 1, 64, [5, 0, 31, 7, 14], [1] * 5),
    "tokens_f32": ("float32", 2, 3, 128, [0, 6, 15, 33], [1] * 4),
    "tokens_f32_64": ("float32", 5, 1, 64, [2, 13], [1, 1]),
    "mixed": ("float16", 2, 2, 64, [0, 13, 16, 30, 7], [3, 20, 0, 2, 40]),
    "prompts": ("bfloat16", 4, 1, 128, [0, 0, 5], [100, 16, 33]),
    "prompts_f32": ("float32", 2, 1, 128, [0, 9], [50, 17]),
    "wide_heads": ("float16", 40, 2, 128, [3, 0], [2, 18]),
    "block_parts": ("bfloat16", 2, 1, 64, [1, 2, 3, 5, 6, 7, 9, 10, 11, 13, 14, 15], [1, 2, 3, 4, 5, 6, 7, 2, 2, 2, 1, 1]),
}


@pytest.mark.parametrize("name", CASES)
def test_plain_rows(name):
    """No norm, no rotation: every code, scale and kept token as the definition has it."""
    dtype, heads, ratio, dim, cached, rows = CASES[name]
    plan, batch, off = setup(dtype, heads, dim, cached, rows)
    for seed, small in ((1, 1.0), (2, 0.05), (3, 30.0)):              # kept tokens as large as the new ones, smaller, larger
        pool = random_pool(plan, seed, small)
        T = int(off[-1]) + 2                                         # two rows of padding
        q, k, v = (du.queries(T, n, dim, dtype, seed=seed + i) for i, n in enumerate((heads * ratio, heads, heads)))
        f, got, _ = fill(plan, off, pool, q, k, v)
        for i, (rowsx, part) in enumerate(((k, "keys"), (v, "values"))):
            want = oracle.fill(rowsx.double().numpy(), *pool[i], off, plan.suffix_tables, plan.suffix_lens)
            same(got[i], want, f"{name} {part}")
        n = int(off[-1])
        assert torch.equal(f.q_out[:n].cpu(), q[:n]) and torch.isnan(f.q_out[n:]).all()


@pytest.mark.parametrize("rotary_dim,interleaved", [(128, False), (128, True), (64, False), (20, False), (50, True), (20, True)])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("single", [True, False])
def test_norm_and_rotation(rotary_dim, interleaved, dtype, single):
    import paper_2405_19888_amd as parrot
    cached, rows = ([3, 0, 16, 200], [1, 1, 1, 1]) if single else ([3, 0, 16], [30, 5, 1])
    plan, batch, off = setup(dtype, 3, 128, cached, rows)
    T = int(off[-1])
    q, k, v = (du.queries(T, n, 128, dtype, seed=i) for i, n in enumerate((6, 3, 3)))
    wq, wk = (1 + 0.1 * du.queries(1, 1, 128, dtype, seed=9 + i)[0, 0] for i in range(2))
    positions = np.concatenate([np.arange(c, c + n) * 37 for c, n in zip(cached, rows)])
    rotary = parrot.make_rotary(rotary_dim, interleaved=interleaved, scaling="yarn", factor=4.0, original_length=4096)
    pool = random_pool(plan, 5)
    f, got, _ = fill(plan, off, pool, q, k, v, positions, rotary, q_norm=wq, k_norm=wk)
    radians, amplitude = drafts_oracle.rotary_frequencies(rotary_dim, scaling="yarn", factor=4.0, original_length=4096)
    y, size = drafts_oracle.rotate(k, positions, radians, interleaved, amplitude, wk, EPS)
    want = oracle.fill(y, *pool[0], off, plan.suffix_tables, plan.suffix_lens)
    assert np.array_equal(got[0][1], want[1])                         # scales (no border is that near at these seeds)
    # a code is off by half a step of the value, and by the key's own error
    err = STEPS * du.F32 * size * float(wk.double().abs().max())
    values = oracle.values(*got[0])
    for row, blk, slot in drafts_oracle.fill_slots(off, plan.suffix_tables, plan.suffix_lens):
        s = oracle.scale(got[0][1][blk])[:, None]
        x = values[blk, :, slot]
        tol = np.maximum(2.0 ** -4 * (np.abs(y[row]) + err[row]), 2.0 ** -10 * s) * (1 + 1e-12) + err[row]
        assert (np.abs(x - y[row]) <= tol).all()
    same(got[1], oracle.fill(v.double().numpy(), *pool[1], off, plan.suffix_tables, plan.suffix_lens), "values")
    yq, sq = drafts_oracle.rotate(q, positions, radians, interleaved, amplitude, wq, EPS)
    tol = du.UNIT[dtype] * np.abs(yq) * 1.01 + STEPS * du.F32 * sq * float(wq.double().abs().max()) + 1e-30
    assert (np.abs(f.q_out.double().cpu().numpy() - yq) <= tol).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_single_rows_have_the_formulas_codes(dtype, interleaved):
    """Of 200000 keys, normalised and rotated, each has the code nearest to its value in 64 bits (in
    fp32 about one in a million has the one beside it)."""
    import paper_2405_19888_amd as parrot
    cached = np.random.default_rng(7).integers(0, 40, 200).tolist()
    plan, batch, off = setup(dtype, 8, 128, cached, [1] * 200)
    k, v = du.queries(200, 8, 128, dtype, seed=1), du.queries(200, 8, 128, dtype, seed=2)
    wk = 1 + 0.1 * du.queries(1, 1, 128, dtype, seed=9)[0, 0]
    positions = np.array(cached) * 311
    rotary = parrot.make_rotary(128, interleaved=interleaved)
    pool = random_pool(plan, 5)
    f, got, _ = fill(plan, off, pool, None, k, v, positions, rotary, k_norm=wk)
    radians, amplitude = drafts_oracle.rotary_frequencies(128)
    y, _ = drafts_oracle.rotate(k, positions, radians, interleaved, amplitude, wk, EPS)
    same(got[0], oracle.fill(y, *pool[0], off, plan.suffix_tables, plan.suffix_lens), "keys")


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows", [1, 7])
def test_values_at_the_borders(dtype, rows):
    """Powers of two, 448 times them and just above, subnormal codes, zeros, ties, and what is no
    finite number."""
    plan, batch, off = setup(dtype, 4, 64, [2, 0], [rows, rows])
    T = int(off[-1])
    k, v = torch.zeros(T, 4, 64, dtype=du.TORCH_DTYPES[dtype]), torch.zeros(T, 4, 64, dtype=du.TORCH_DTYPES[dtype])
    top = torch.tensor([448.0, 450.0, 1.0, 0.0]).to(k.dtype)          # the heads' largest
    k[0, :, 0], v[T - 1, :, 5] = top, -top
    line = torch.cat([2.0 ** -torch.arange(24).double(), 3 * 2.0 ** -torch.arange(16).double(), torch.tensor([17.0, 19.0, 21.0, -17.0])])
    k[0, :, 10:10 + len(line)] = line.to(k.dtype)
    v[T - 1, 0, 10:10 + len(line)] = line.to(k.dtype)
    k[0, 1, 60], k[0, 1, 61], k[0, 1, 62] = float("nan"), float("inf"), -float("inf")
    v[0, 2, 3] = float("inf")
    pool = random_pool(plan, 3)
    f, got, _ = fill(plan, off, pool, None, k, v)
    for i, x in enumerate((k, v)):
        same(got[i], oracle.fill(x.double().numpy(), *pool[i], off, plan.suffix_tables, plan.suffix_lens), "kv"[i])


def test_largest_and_smallest_numbers():
    plan, batch, off = setup("float32", 3, 64, [0, 3], [2, 1])
    k, v = torch.zeros(3, 3, 64), torch.zeros(3, 3, 64)
    k[:, 0, 1], k[:, 1, 1], k[:, 2, 1] = 3.4e38, 1e-38, 1e-45
    v[0, 0, 0], v[1, 1, 0], v[2, 2, 0] = -3.3e38, 2.0 ** -126, 2.0 ** -149
    pool = random_pool(plan, 3, 1e-12)
    f, got, _ = fill(plan, off, pool, None, k, v)
    for i, x in enumerate((k, v)):
        same(got[i], oracle.fill(x.double().numpy(), *pool[i], off, plan.suffix_tables, plan.suffix_lens), "kv"[i])


def test_scales_grow_token_by_token():
    """Thirty decode steps of one request, rows growing and shrinking: every step's pool as the
    definition has it, after the step before."""
    rng = np.random.default_rng(0)
    plan, batch, off = setup("bfloat16", 2, 64, [0], [30])
    pool = random_pool(plan, 1)
    for p in range(30):
        from dataclasses import replace
        step = replace(plan, suffix_lens=np.array([p + 1], dtype=np.int32))
        k, v = (du.queries(1, 2, 64, "bfloat16", seed=p + s) * 2.0 ** int(rng.integers(-6, 7)) for s in (0, 100))
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
        f, got, _ = fill(step, np.array([0, 1], dtype=np.int32), pool, None, k, v)
        want = [oracle.fill(x.double().numpy(), *pool[i], [0, 1], step.suffix_tables, step.suffix_lens) for i, x in enumerate((k, v))]
        for i in range(2):
            same(got[i], want[i], f"step {p}")
        pool = want


def test_separate_rows_and_queries_in_place():
    import paper_2405_19888_amd as parrot
    plan, batch, off = setup("float16", 2, 128, [5, 0], [9, 20])
    T = int(off[-1])
    q, k, v = (du.queries(T, n, 128, "float16", seed=i) for i, n in enumerate((4, 2, 2)))
    pool = random_pool(plan, 2)
    f, got, t = fill(plan, off, pool, q, k, v, fused=False)
    for i, x in enumerate((k, v)):
        same(got[i], oracle.fill(x.double().numpy(), *pool[i], off, plan.suffix_tables, plan.suffix_lens), "kv"[i])
    rotary = parrot.make_rotary(128)
    pos = torch.arange(T, dtype=torch.int32).cuda()
    args = [t[x] for x in ("query_offsets", "suffix_tables", "suffix_lens")]
    mine = q.cuda()
    parrot.parrot_cache8_fill(f.problem, T, 20, 4, rotary, mine, t["k_rows"], t["v_rows"], None, None, pos, *args, mine, t["suffix"])
    apart = parrot.cache8_fill(q.cuda(), t["k_rows"], t["v_rows"], pos, args[0], t["suffix"], *args[1:], rotary=rotary)
    assert torch.equal(mine, apart)


def test_bounds_larger_than_the_batch():
    """One bound handle serves shorter calls: max_query_rows above every request's rows gives the
    same pool, single tokens included."""
    plan, batch, off = setup("float16", 3, 128, [5, 15, 0, 30], [1, 1, 1, 1])
    q, k, v = (du.queries(4, n, 128, "float16", seed=i) for i, n in enumerate((3, 3, 3)))
    pool = random_pool(plan, 2, 0.1)
    one = fill(plan, off, pool, q, k, v)[1]
    many = fill(plan, off, pool, q, k, v, max_rows=6)[1]
    for a, b in zip(one, many):
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_many_requests_find_their_units():
    rng = np.random.default_rng(1)
    rows = rng.integers(0, 40, 200).tolist()
    cached = rng.integers(0, 40, 200).tolist()
    cached = [c + (c + n == 0) for c, n in zip(cached, rows)]
    plan, batch, off = setup("float16", 1, 64, cached, rows)
    T = int(off[-1])
    k, v = (du.queries(T, 1, 64, "float16", seed=i) for i in range(2))
    pool = random_pool(plan, 2)
    _, got, _ = fill(plan, off, pool, None, k, v)
    for i, x in enumerate((k, v)):
        same(got[i], oracle.fill(x.double().numpy(), *pool[i], off, plan.suffix_tables, plan.suffix_lens), "kv"[i])


def test_fill_then_attention_in_one_graph():
    """Decode steps as an engine runs them: fill, plan and attention captured once, replayed over
    growing lengths with new rows, against the same calls made eagerly on a copy of the pool."""
    import paper_2405_19888_amd as parrot
    heads, ratio, dim, R = 2, 4, 128, 3
    plan, batch, off = setup("bfloat16", heads, dim, [28, 14, 2], [6, 6, 6])
    lens = torch.tensor([29, 15, 3], dtype=torch.int32, device="cuda")
    one = np.arange(R + 1, dtype=np.int32)
    (ck, bk), (cv, bv) = random_pool(plan, 4)
    pools = [cu.device_pools(ck, oracle.value_order(cv), np.stack([bk, bv], -1)) for _ in range(2)]
    x = torch.zeros(R, (ratio + 2) * heads * dim, dtype=torch.bfloat16, device="cuda")
    parts = [y.unflatten(1, (-1, dim)) for y in x.split([ratio * heads * dim, heads * dim, heads * dim], 1)]
    t = dict(q_rows=parts[0], k_rows=parts[1], v_rows=parts[2], query_offsets=torch.from_numpy(one).cuda(), suffix_lens=lens,
             suffix_tables=torch.from_numpy(plan.suffix_tables).cuda(), positions=lens - 1,
             group_ids=torch.full((R,), -1, dtype=torch.int32, device="cuda"))
    prob = parrot.problem_from_host(num_heads=heads, head_dim=dim, block_size=16, dtype=torch.bfloat16, sm_scale=dim ** -0.5,
                                    group_ids=[-1] * R, prefix_lens=[], suffix_lens=plan.suffix_lens, prefix_table_stride=0,
                                    suffix_table_stride=plan.suffix_tables.shape[1], num_suffix_blocks=plan.num_blocks,
                                    num_prefix_blocks=0)
    rows = parrot.make_tree_rows(R, 1, 0, heads * ratio)
    rotary = parrot.make_rotary(dim)

    def step(pool):
        f = parrot.Cache8Filler(prob, R, 1, heads * ratio, rotary=rotary)
        planner = parrot.Cache8Planner(prob, rows)
        dec = parrot.Cache8Decoder(planner)
        a = {**t, "suffix": pool}
        calls = [f.bind(a), planner.bind(a), dec.bind({**a, "q_rows": f.q_out})]
        return f, dec, calls

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        kept = step(pools[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            captured = [kept[0].bind({**t, "suffix": pools[0]})]
            captured[0]()
            planner = kept[1].planner
            planner.bind({**t, "suffix": pools[0]})()
            kept[1].bind({**t, "suffix": pools[0], "q_rows": kept[0].q_out})()
    eager = step(pools[1])
    for i in range(5):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)).to(x.dtype))
        t["positions"].copy_(lens - 1)
        torch.cuda.synchronize()
        [c() for c in eager[2]]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in pools[0]:
            assert torch.equal(pools[0][name].view(torch.uint8), pools[1][name].view(torch.uint8)), (i, name)
        assert torch.equal(kept[1].out, eager[1].out) and torch.equal(kept[1].lse, eager[1].lse), i
        lens += 1
