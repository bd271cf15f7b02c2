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
