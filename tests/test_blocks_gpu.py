"""Copies of cache blocks: pools of several sizes and types, skipped pairs, many pools, graphs."""
import numpy as np
import pytest
import torch

from oracle import cache8 as oracle

pytestmark = pytest.mark.gpu


def pools_of(blocks, shapes, seed=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for dtype, *shape in shapes:
        x = torch.randint(0, 256, (blocks, *shape, dtype.itemsize), generator=g, dtype=torch.uint8)
        out.append(x.view(dtype).squeeze(-1).cuda() if dtype.itemsize > 1 else x.squeeze(-1).cuda())
    return out


def as_bytes(x):
    return x.contiguous().view(torch.uint8).reshape(x.shape[0], -1).cpu().numpy()


SHAPES = {
    "layer_of_8_bits": [(torch.uint8, 4, 16, 128), (torch.uint8, 4, 2, 4, 16, 4, 4), (torch.uint8, 4, 2)],
    "half_precision": [(torch.float16, 5, 16, 64)] * 4,
    "floats": [(torch.float32, 3, 16, 128), (torch.float32, 40, 16, 128)],
    "odd_scales": [(torch.uint8, 1, 2), (torch.uint8, 3, 2), (torch.uint8, 7, 2)],
    "large_block": [(torch.float32, 64, 16, 128)],
    "300_pools": [(torch.uint8, 1, 16, 64)] * 300,
}


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("copies", [1, 7])
def test_copies(name, copies):
    import paper_2405_19888_amd as parrot
    pools = pools_of(20, SHAPES[name])
    ids = np.random.default_rng(copies).permutation(20)
    src, dst = ids[:copies], ids[copies:2 * copies]
    want = oracle.copy_blocks([as_bytes(x) for x in pools], src, dst)
    parrot.copy_blocks(pools, src, dst)
    for x, y in zip(pools, want):
        assert np.array_equal(as_bytes(x), y)


def test_one_source_for_several_and_skipped_pairs():
    import paper_2405_19888_amd as parrot
    pools = pools_of(12, SHAPES["layer_of_8_bits"])
    src, dst = [3, 3, -1, 5, 4, 40, 6], [0, 1, 2, -1, 7, 8, 12]
    want = oracle.copy_blocks([as_bytes(x) for x in pools], src, dst)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    parrot.copy_blocks(pools, ints(src), ints(dst))
    torch.cuda.synchronize()
    for x, y in zip(pools, want):
        assert np.array_equal(as_bytes(x), y)


def test_bound_call_on_a_stream_and_in_a_graph():
    import paper_2405_19888_amd as parrot
    pools = pools_of(30, SHAPES["layer_of_8_bits"])
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    src, dst = ints([-1] * 5), ints([-1] * 5)
    copier = parrot.BlockCopier(pools, 5)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            copier.bind(src, dst)()
    for a, b in (([1, 2, 3, 4, 5], [11, 12, 13, 14, 15]), ([11, 15, -1, -1, -1], [0, 29, -1, -1, -1]), ([-1] * 5, [-1] * 5)):
        want = oracle.copy_blocks([as_bytes(x) for x in pools], a, b)
        src.copy_(ints(a))
        dst.copy_(ints(b))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(pools, want):
            assert np.array_equal(as_bytes(x), y)


def test_blocks_beyond_four_gigabytes():
    import paper_2405_19888_amd as parrot
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GiB free")
    pool = torch.zeros(9000, 1 << 19, dtype=torch.uint8, device="cuda")          # 4.7e9 bytes
    pool[8999] = 7
    parrot.copy_blocks([pool], [8999], [8500])
    assert bool((pool[8500] == 7).all()) and not bool(pool[8501].any()) and not bool(pool[8499].any())


def test_decode_steps_of_forks():
    """An engine's steps over the store and two layers held in 8 bits: contexts on a prefix fork, append, are
    truncated, freed and compacted; each step copies what the store owes, fills the new rows and attends.
    Every block is the definition's, each context reads its own tokens, outputs are within their bound."""
    from types import SimpleNamespace

    import cache8_util as cu
    import paper_2405_19888_amd as parrot
    from paper_2405_19888_amd.context import ContextStore
    H, HQ, D, N = 2, 6, 64, 60
    gen, rng = torch.Generator().manual_seed(5), np.random.default_rng(2)
    st = ContextStore(16, N)
    layers = [parrot.cache8_pools(N, H, D) for _ in range(2)]
    pools = [x for layer in layers for x in layer.values()]
    model = [[(np.zeros((N, H, 16, D), np.uint8), np.zeros((N, H), np.uint8)) for _ in "kv"] for _ in layers]
    truth = {}                                           # per context and layer: its own keys' and values' rows
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()

    def write(layer, k, v, off, tables, lens, q=None):
        out = parrot.cache8_fill(None if q is None else q.cuda(), k.cuda(), v.cuda(), None, t(off), layers[layer], t(tables), t(lens))
        for i, x in enumerate((k, v)):
            model[layer][i] = oracle.fill(x.double().numpy(), *model[layer][i], off, tables, lens)
        return out

    def draw(rows, heads):
        size = torch.exp2(torch.randint(-3, 4, (rows, 1, 1), generator=gen).float())
        return (torch.randn(rows, heads, D, generator=gen) * size).to(torch.bfloat16)

    prompt = list(range(40))
    ctxs = [st.fill(prompt + [100 + i] * n, [40]) for i, n in enumerate((21, 5, 47))] + [st.fill([7] * 30)]
    batch = st.build_batch(ctxs)
    off = np.concatenate([[0], np.cumsum(batch.suffix_lens)]).astype(np.int32)
    for layer in range(2):
        write(layer, draw(40, H), draw(40, H), np.array([0, 40], np.int32), batch.prefix_tables, batch.prefix_lens)
        k, v = draw(int(off[-1]), H), draw(int(off[-1]), H)
        write(layer, k, v, off, batch.suffix_tables, batch.suffix_lens)
        for r, c in enumerate(ctxs):
            truth[c, layer] = [list(x[off[r]:off[r + 1]].double().numpy()) for x in (k, v)]
    a, b, c, d = ctxs

    def fork(x):
        y = st.fork(x)
        for layer in range(2):
            truth[y, layer] = [list(z) for z in truth[x, layer]]
        return y

    copied = 0
    for step in range(8):
        if step == 0:
            ctxs += [fork(a), fork(a), fork(c)]
        if step == 2:
            st.free(a)
            ctxs.remove(a)
            ctxs += [fork(b), fork(d)]
        if step == 3:
            st.truncate(d, 17)
            st.truncate(c, 34)
            for layer in range(2):
                for z in truth[d, layer]:
                    del z[17:]
                for z in truth[c, layer]:
                    del z[34:]
        if step == 5:
            st.free(b)
            ctxs.remove(b)
            st.free(d)
            ctxs.remove(d)
            assert st.compact() > 0
        rows = [int(x) for x in rng.integers(1, 4 if step % 2 else 2, len(ctxs))]
        for x, n in zip(ctxs, rows):
            for _ in range(n):
                st.append(x)
        src, dst = st.take_copies()
        copied += len(src)
        parrot.copy_blocks(pools, src.tolist(), dst.tolist())
        for layer in model:
            for codes, byte in layer:
                codes[dst], byte[dst] = codes[src].copy(), byte[src].copy()
        batch = st.build_batch(ctxs)
        off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        plan = SimpleNamespace(head_dim=D, dtype="bfloat16", sm_scale=D ** -0.5, nested=False, prefix_parents=None,
                               **{x: getattr(batch, x) for x in ("group_ids", "prefix_lens", "suffix_lens", "prefix_tables", "suffix_tables")})
        for layer in range(2):
            k, v, q = draw(int(off[-1]), H), draw(int(off[-1]), H), draw(int(off[-1]), HQ)
            turned = write(layer, k, v, off, batch.suffix_tables, batch.suffix_lens, q)
            assert torch.equal(turned.cpu(), q)
            used = sorted({int(x) for r in range(len(ctxs)) for x in batch.suffix_tables[r][:-(-int(batch.suffix_lens[r]) // 16)]} |
                          {int(x) for x in batch.prefix_tables[0][:3]})
            got = parrot.cache8_values(layers[layer], torch.tensor(used).cuda())
            want = [oracle.values(*x) for x in model[layer]]
            for g, w in zip(got, want):
                assert np.array_equal(g.double().cpu().numpy(), w[used]), (step, layer)
            for r, x in enumerate(ctxs):
                for i, new in enumerate((k, v)):
                    truth[x, layer][i] += list(new[off[r]:off[r + 1]].double().numpy())
                    rows_x, tab = np.array(truth[x, layer][i]), batch.suffix_tables[r]
                    assert len(rows_x) == st.own_tokens(x)
                    p = np.arange(len(rows_x))
                    held = want[i][tab[p // 16], :, p % 16]
                    # half a code's step, and where a scale grew those of its least codes (each at most half the next)
                    size = oracle.scale(model[layer][i][1][tab[p // 16]])[..., None]
                    assert (np.abs(held - rows_x) <= 2.0 ** -4 * np.abs(rows_x) + 2.0 ** -9 * size).all(), (step, layer, x)
            out, lse = parrot.cache8_attention(q.cuda(), t(off), layers[layer], layers[layer], t(batch.prefix_tables), t(batch.prefix_lens),
                                               t(batch.suffix_tables), t(batch.suffix_lens), t(batch.group_ids))
            cu.check(plan, want, q, off, out, lse, what=f"step {step} layer {layer}")
    assert copied >= 6
