"""One-call forms on a stream of their own: the sizes they read, and the memory they allocate,
belong to that stream."""
import numpy as np
import pytest
import torch

import drafts_util as du

pytestmark = pytest.mark.gpu


def late(s, targets):
    """Queues work on s and then the targets' values; they hold less until then."""
    held = [x.clone() for x in targets]
    for x in targets:
        x.clamp_(max=1)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        x = torch.randn((4096, 4096), device="cuda")
        for _ in range(20):
            x = (x @ x).clamp_(-1, 1)
        for t, h in zip(targets, held):
            t.copy_(h)
    return held                                        # (read when the stream gets there)


def on_stream(call, targets, handle):
    """The call's results on a busy side stream, given as a stream or by its handle."""
    s = torch.cuda.Stream()
    held = late(s, targets)
    got = call(s.cuda_stream if handle else s)
    s.synchronize()
    del held
    return got


def step():
    rows, cached = [5, 8], [10, 40]
    plan = du.tree_plan("float16", 2, 64, [0, 0], [33], cached, rows)
    batch, off = du.make_batch(plan), du.offsets_of(rows)
    dev = batch.to("cuda")
    up = du.random_trees(np.random.default_rng(4), rows)
    ints = lambda x: torch.tensor(np.asarray(x, dtype=np.int32)).cuda()
    dev.update(off=ints(off), up=ints(up), q=du.queries(13, 4, 64, "float16").cuda(),
               k=du.queries(13, 2, 64, "float16", seed=1).cuda(), v=du.queries(13, 2, 64, "float16", seed=2).cuda(),
               tokens=ints(np.zeros(13)), roots=ints([0, 0]), rows=ints([0, 2, -1, -1, -1, 1, 3, 4] + [-1] * 5), lens=ints([2, 3]))
    return dev


def forms(d):
    import paper_2405_19888_amd as parrot
    cache = (d["k_pool"], d["v_pool"], d["suffix_tables"], d["suffix_lens"])
    pools = (d["k_pool"], d["v_pool"], d["k_pool"], d["v_pool"], d["prefix_tables"], d["prefix_lens"], d["suffix_tables"],
             d["suffix_lens"], d["group_ids"])
    return {
        "fill": lambda s: parrot.rotary_fill(d["q"], d["k"], d["v"], d["tokens"], d["off"], *cache,
                                             rotary=parrot.make_rotary(64), stream=s),
        "tree": lambda s: parrot.tree_decode(d["q"], d["off"], d["up"], *pools, stream=s),
        "accept": lambda s: parrot.tree_accept(d["off"], d["up"], d["tokens"], d["tokens"], d["roots"], stream=s),
        "decode": lambda s: parrot.shared_prefix_decode(d["q"][:2, :2].contiguous(), *pools, sm_scale=0.125, stream=s),
        "prefill": lambda s: parrot.shared_prefix_prefill(d["q"][:, :2].contiguous(), d["off"], *pools, sm_scale=0.125, stream=s),
        "commit": lambda s: parrot.tree_commit(d["off"], d["rows"], d["lens"], *cache, stream=s),
    }


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", ["fill", "tree", "accept", "commit", "decode", "prefill"])
def test_sizes_and_memory_are_the_streams(name, handle):
    d, fresh = step(), step()
    want = forms(fresh)[name](None)
    torch.cuda.synchronize()
    got = on_stream(forms(d)[name], [d["off"], d["suffix_lens"]], handle)
    tensors = lambda x: [x] if isinstance(x, torch.Tensor) else list(x)
    for a, b in zip(tensors(got), tensors(want)):
        assert torch.equal(a, b)
    for x in ("k_pool", "v_pool"):
        assert torch.equal(torch.nan_to_num(d[x], 9.0), torch.nan_to_num(fresh[x], 9.0))
    # dropped results stay the side stream's
    like = [(x.shape, x.dtype, x.data_ptr()) for x in tensors(got)]
    del got
    new = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype, _ in like]
    assert not {x.data_ptr() for x in new} & {p for _, _, p in like}


def test_default_stream_by_its_handle():
    d = step()
    want = forms(d)["tree"](None)
    got = forms(d)["tree"](0)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
