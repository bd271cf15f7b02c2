"""GPU parity of accept and commit (integers and copied bytes: equal), and a whole
drafting step over the context store: fill, tree attention, accept, commit."""
import numpy as np
import pytest
import torch

import drafts_util as du
from drafts_util import oracle

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32)).cuda()


def accept(off, up, draft, target, root, T=None):
    import paper_2405_19888_amd as parrot
    T = len(draft) if T is None else T
    rows = parrot.make_tree_rows(T, max(1, int(np.diff(off).max())), 0, 1)
    taken, lens, follow = (torch.full((n,), -77, dtype=torch.int32).cuda() for n in (T, len(root), len(root)))
    parrot.parrot_tree_accept(len(root), rows, ints(off), None if up is None else ints(up), ints(draft), ints(target),
                              ints(root), taken, lens, follow)
    torch.cuda.synchronize()
    return taken.cpu().numpy(), lens.cpu().numpy(), follow.cpu().numpy()


@pytest.mark.parametrize("vocabulary", [2, 5, 1000])
@pytest.mark.parametrize("trees", [True, False])
def test_accept(vocabulary, trees):
    """Small vocabularies make long paths and siblings with the same token."""
    rng = np.random.default_rng(vocabulary)
    rows = [int(x) for x in rng.integers(0, 129, 70)] + [128, 1, 0, 64, 65]
    off = du.offsets_of(rows)
    T = int(off[-1])
    up = du.random_trees(rng, rows, spread=6, roots=2)
    draft, target = rng.integers(0, vocabulary, T + 3), rng.integers(0, vocabulary, T + 3)
    root = rng.integers(0, vocabulary, len(rows))
    up = np.concatenate([up, [0, 0, 0]])
    got = accept(off, up if trees else None, draft, target, root)
    want = oracle.tree_accept(off, up if trees else None, draft, target, root)
    assert (got[0][T:] == -77).all(), "padding was written"
    for g, w in zip((got[0][:T], *got[1:]), (want[0][:T], *want[1:])):
        assert np.array_equal(g, w)


def test_accept_whole_chain_and_nothing():
    tokens = np.arange(128)
    got = accept([0, 128], None, tokens, tokens + 1, [0])
    assert got[1][0] == 128 and np.array_equal(got[0], np.arange(128)) and got[2][0] == 128
    got = accept([0, 128], None, tokens, tokens + 1, [5])
    assert got[1][0] == 0 and (got[0] == -1).all() and got[2][0] == 5
    # parents that break the rules are never followed
    got = accept([0, 3], [2, 5, -9], [1, 1, 1], [1, 1, 1], [1])
    assert got[1][0] == 0
    # negative token ids are tokens like any other
    got = accept([0, 2], [-1, 0], [-1, -3], [-3, 4], [-1])
    assert got[1][0] == 2 and got[2][0] == 4


def test_accept_without_rows():
    got = accept([0, 0, 0], None, [], [], [3, 4], T=0)
    assert (got[1] == 0).all() and np.array_equal(got[2], [3, 4])


@pytest.mark.parametrize("dtype,heads,dim", [("float16", 32, 128), ("bfloat16", 5, 64), ("float32", 9, 128),
                                             ("float32", 1, 64)])
def test_commit(dtype, heads, dim):
    """Paths whose moved rows are other rows' targets, none, one and all rows."""
    import paper_2405_19888_amd as parrot
    rng = np.random.default_rng(heads)
    rows = [int(x) for x in rng.integers(1, 60, 11)] + [128, 128, 5, 7, 0]
    cached = [int(x) for x in rng.integers(0, 50, 13)] + [16, 0, 33]
    plan = du.tree_plan(dtype, heads, dim, [-1] * 16, [], cached, rows, seed=heads)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    taken, lens = np.full(int(off[-1]), -1), []
    for r, n in enumerate(rows):
        m = int(rng.integers(0, n + 1)) if r < 11 else {11: 128, 12: 127, 13: 0, 14: 1}.get(r, 0)
        path = np.sort(rng.choice(n, m, replace=False)) if r != 12 else np.arange(1, 128)
        taken[off[r]:off[r] + m] = path
        lens.append(m)
    dev = batch.to("cuda")
    from gpu_util import problem_for
    prob = problem_for(plan)
    counts = parrot.make_tree_rows(int(off[-1]), 128, 0, 1)
    out = torch.full((16,), -1, dtype=torch.int32).cuda()
    parrot.parrot_tree_commit(prob, counts, ints(off), ints(taken), ints(lens), dev["suffix_tables"],
                              dev["suffix_lens"], dev["k_pool"], dev["v_pool"], out)
    torch.cuda.synchronize()
    moves, after = oracle.tree_commit(off, taken, lens, plan.suffix_tables, plan.suffix_lens)
    for pool, got in ((batch.k_pool, dev["k_pool"]), (batch.v_pool, dev["v_pool"])):
        want = pool.clone()
        for (a, i), (b, j) in moves:
            want[b, :, j] = pool[a, :, i]
        assert torch.equal(torch.nan_to_num(got.cpu(), 9.0), torch.nan_to_num(want, 9.0))
    assert np.array_equal(out.cpu().numpy(), after)


def test_drafting_step_over_the_store():
    """Two steps of three contexts on one cached prefix: drafted trees are filled,
    attended to, accepted and committed on the device, the store follows, and a decode
    over the committed cache equals one over a cache filled in order."""
    import paper_2405_19888_amd as parrot
    from paper_2405_19888_amd.context import ContextStore
    H, HQ, D, V = 2, 4, 64, 3
    rng = np.random.default_rng(8)
    gen = torch.Generator().manual_seed(3)
    draw = lambda *s: torch.randn(*s, generator=gen).half().cuda()
    store = ContextStore(16, 64)
    prompt = list(range(40))
    ctxs = [store.fill(prompt + [100 + i] * (7 * i + 1), [40]) for i in range(3)]
    kp, vp = draw(64, H, 16, D), draw(64, H, 16, D)
    rotary = parrot.make_rotary(D)
    spare = {}                                             # rows by token, as a model would compute them
    for step in range(2):
        cached = [store.own_tokens(c) for c in ctxs]
        rows = [int(x) for x in rng.integers(3, 9, 3)]
        for c, n in zip(ctxs, rows):
            for _ in range(n):
                store.append(c)
        b = store.build_batch(ctxs)
        off = du.offsets_of(rows)
        T = int(off[-1])
        up = du.random_trees(rng, rows, spread=3)
        depth = np.concatenate([[len(oracle.tree_path(up[off[r]:off[r + 1]], j)) - 1 for j in range(n)]
                                for r, n in enumerate(rows)])
        positions = 40 + np.repeat(cached, rows) + depth
        q, k, v = draw(T, HQ, D), draw(T, H, D), draw(T, H, D)
        dev = {x: torch.from_numpy(getattr(b, x)).cuda() for x in
               ("group_ids", "suffix_lens", "suffix_tables", "prefix_lens", "prefix_parents", "prefix_tables")}
        dev.update(q_rows=q, k_rows=k, v_rows=v, positions=ints(positions), query_offsets=ints(off),
                   tree_parents=ints(up), k_pool=kp, v_pool=vp)
        prob = parrot.problem_from_host(
            num_heads=H, head_dim=D, block_size=16, dtype=torch.float16, sm_scale=D ** -0.5, group_ids=b.group_ids,
            prefix_lens=b.prefix_lens, suffix_lens=b.suffix_lens, prefix_table_stride=b.prefix_tables.shape[1],
            suffix_table_stride=b.suffix_tables.shape[1], num_prefix_blocks=64, num_suffix_blocks=64)
        counts = parrot.tree_rows_from_host(off, b.group_ids, len(b.prefix_lens), HQ)
        before_k, before_v = kp.clone(), vp.clone()
        filler = parrot.RotaryFiller(prob, T, max(rows), HQ, rotary=rotary)
        dec = parrot.TreeDecoder(prob, counts)
        ver = parrot.TreeVerifier(prob, counts)
        dev["draft_tokens"], dev["target_tokens"] = ints(rng.integers(0, V, T)), ints(rng.integers(0, V, T))
        dev["root_tokens"] = ints(rng.integers(0, V, 3))
        # the whole step on one stream, nothing waits between
        filler.bind(dev)()
        dec.bind(dict(dev, q_rows=filler.q_out))()
        ver.bind_accept(dev)()
        ver.bind_commit(dev)()
        torch.cuda.synchronize()

        # attention, against the cache as the fill left it
        filled_k, filled_v = before_k.cpu(), before_v.cpu()
        radians, amplitude = oracle.rotary_frequencies(D)
        turned = torch.from_numpy(oracle.rotate(k.cpu(), positions, radians, False, amplitude)[0]).half()
        for row, blk, at in oracle.fill_slots(off, b.suffix_tables, b.suffix_lens):
            filled_k[blk, :, at], filled_v[blk, :, at] = turned[row], v[row].cpu()
        ref, rlse, spread, noise = oracle.shared_prefix_tree(
            filler.q_out.cpu(), off, up, filled_k, filled_v, filled_k, filled_v, b.prefix_tables, b.prefix_lens,
            b.suffix_tables, b.suffix_lens, b.group_ids, D ** -0.5)
        # (keys rotated by the oracle may round to the neighbouring half: 2^-11 of a logit more)
        tol = du.out_tolerance("float16", ref, spread, noise, 100, D) + 2 * 2.0 ** -11 * noise[..., None] * spread
        assert (np.abs(dec.out.double().cpu().numpy() - ref) <= tol).all()
        want = oracle.tree_accept(off, up, dev["draft_tokens"].cpu().numpy(), dev["target_tokens"].cpu().numpy(),
                                  dev["root_tokens"].cpu().numpy())
        assert np.array_equal(ver.accept_rows.cpu().numpy(), want[0])
        assert np.array_equal(ver.next_tokens.cpu().numpy(), want[2])

        # the committed cache holds the accepted rows in order; the store drops the rest
        lens = ver.committed_lens.cpu().numpy()
        assert np.array_equal(lens, np.array(cached) + want[1])
        for r, c in enumerate(ctxs):
            store.truncate(c, int(lens[r]))
            assert store.own_tokens(c) == lens[r]
            for i in range(want[1][r]):
                p, row = cached[r] + i, int(off[r] + want[0][off[r] + i])
                blk = int(b.suffix_tables[r][p // 16])
                assert torch.equal(vp[blk, :, p % 16], v[row])
                assert (kp[blk, :, p % 16].cpu().double() - turned[row].double()).abs().max() <= 2.0 ** -10 * 8
    for c in ctxs:
        store.free(c)
    assert store.free_blocks == 64
