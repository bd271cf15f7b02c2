"""Caches held in 8 bits on the host: refusals before any device work, sizes, the Python forms'
checks, and pins of the oracle the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2405_19888_amd as parrot
from oracle import cache8 as oracle
from paper_2405_19888_amd import binding as B
from test_drafts import FAKE, addresses, fill_rows, problem

FILL = ["q", "k", "v", "q_norm", "k_norm", "positions", "query_offsets", "suffix_block_tables", "suffix_lens", "q_out"]
PLAN = ["query_offsets", "prefix_lens", "prefix_parents", "suffix_lens", "group_ids", "plan"]
POOL = ["k", "v", "scales"]


def pool(base, **over):
    vals = {n: FAKE + base + 4096 * i for i, n in enumerate(POOL)}
    vals.update(over)
    return B.ParrotCache8(*(vals[n] for n in POOL))


def fill(lib, prob=None, rows=None, rotary=None, suffix=None, **over):
    prob, rows = prob or problem(), rows or fill_rows()
    suffix = pool(1 << 18) if suffix is None else suffix
    return lib.parrot_cache8_fill(ctypes.byref(prob), ctypes.byref(rows), rotary, *addresses(FILL, over),
                                  ctypes.byref(suffix) if suffix else None, None, None)


def plan(lib, prob=None, rows=None, size=1 << 40, **over):
    prob, rows = prob or problem(), rows or parrot.make_tree_rows(20, 10, 20, 8)
    return lib.parrot_cache8_plan(ctypes.byref(prob), ctypes.byref(rows), *addresses(PLAN, over), size, None)


ATTEND = ["q", "query_offsets", "ptab", "plen", "prefix_parents", "stab", "slen", "gid", "plan", "out", "lse", "ws"]


def attend(lib, prob=None, rows=None, plan_bytes=1 << 40, room=1 << 45, prefix=None, suffix=None, **over):
    prob, rows = prob or problem(), rows or parrot.make_tree_rows(20, 10, 20, 8)
    prefix = pool(1 << 17) if prefix is None else prefix
    suffix = pool(1 << 18) if suffix is None else suffix
    v = dict(zip(ATTEND, addresses(ATTEND, {})))
    v.update(over)
    ref = lambda x: ctypes.byref(x) if x else None
    return lib.parrot_cache8_attention(ctypes.byref(prob), ctypes.byref(rows), v["q"], v["query_offsets"], ref(prefix),
                                       ref(suffix), *(v[n] for n in ATTEND[2:9]), plan_bytes, v["out"], v["lse"], v["ws"],
                                       room, None, None)


def refused(status, msg, want=B.PARROT_ERR_INVALID_ARGUMENT):
    assert status == want, B.parrot_last_error()
    assert msg in B.parrot_last_error(), B.parrot_last_error()


def test_struct_layouts():
    assert ctypes.sizeof(B.ParrotCache8) == 24 and ctypes.sizeof(B.ParrotBlockPool) == 16


def test_fill_pointers(parrot_lib):
    for n in FILL:
        if n not in ("q_norm", "k_norm", "positions"):
            refused(fill(parrot_lib, **{n: None}), "NULL")
        if n != "positions":
            refused(fill(parrot_lib, **{n: FAKE + 1}), "aligned")
    rot = ctypes.byref(parrot.make_rotary(64))
    for bad in (None, FAKE + 2):
        assert fill(parrot_lib, rotary=rot, positions=bad) == B.PARROT_ERR_INVALID_ARGUMENT
    refused(fill(parrot_lib, suffix=False), "suffix is NULL")
    for n in POOL:
        refused(fill(parrot_lib, suffix=pool(1 << 18, **{n: None})), f"suffix->{n} is NULL")
        refused(fill(parrot_lib, suffix=pool(1 << 18, **{n: FAKE + 2})), f"suffix->{n}")
    refused(fill(parrot_lib, suffix=pool(0, v=FAKE)), "same pool")


@pytest.mark.parametrize("over,msg", [
    (dict(num_query_rows=-1), "num_query_rows"), (dict(max_query_rows=0), "max_query_rows"),
    (dict(max_query_rows=301), "max_query_rows"), (dict(num_query_heads=0), "num_query_heads"),
    (dict(norm_eps=-1.0), "norm_eps"), (dict(q_stride=1016), "q_stride"), (dict(k_stride=516), "16 bytes"),
    (dict(v_stride=-512), "v_stride")])
def test_fill_refusals(parrot_lib, over, msg):
    refused(fill(parrot_lib, rows=fill_rows(**over)), msg)


def test_fill_more_refusals(parrot_lib):
    refused(fill(parrot_lib, prob=problem(head_dim=64), rotary=ctypes.byref(parrot.make_rotary(128))), "head_dim")
    refused(fill(parrot_lib, prob=problem(head_dim=80)), "head_dim", B.PARROT_ERR_UNSUPPORTED)
    refused(fill(parrot_lib, prob=problem(block_size=32)), "block_size", B.PARROT_ERR_UNSUPPORTED)
    refused(fill(parrot_lib, rows=fill_rows(q_stride=2048), q=FAKE, q_out=FAKE), "q_out")
    assert fill(parrot_lib, rows=fill_rows(num_query_rows=0), k=None) == B.PARROT_OK


def test_attention_pointers(parrot_lib):
    for n in PLAN:
        if n != "prefix_parents":
            refused(plan(parrot_lib, **{n: None}), "NULL")
        refused(plan(parrot_lib, **{n: FAKE + 1}), "aligned")
    for n in ATTEND:
        if n != "prefix_parents":
            refused(attend(parrot_lib, **{n: None}), "NULL")
        refused(attend(parrot_lib, **{n: FAKE + 1}), "aligned")
    refused(attend(parrot_lib, plan=FAKE + 128), "plan")
    for which in ("prefix", "suffix"):
        refused(attend(parrot_lib, **{which: False}), f"{which} is NULL")
        for n in POOL:
            refused(attend(parrot_lib, **{which: pool(1 << 18, **{n: FAKE + 2})}), f"{which}->{n}")
    refused(attend(parrot_lib, q=FAKE, out=FAKE), "out is q")


@pytest.mark.parametrize("rows,msg,status", [
    ((-1, 10, 20, 8), "num_query_rows", 1), ((20, 0, 20, 8), "max_query_rows", 1), ((20, 301, 20, 8), "max_query_rows", 1),
    ((20, 10, 21, 8), "max_group_rows", 1), ((20, 10, -1, 8), "max_group_rows", 1), ((20, 10, 20, 6), "multiple", 1),
    ((20, 10, 20, 0), "multiple", 1), ((1 << 30, 128, 20, 8), "2^31", 2)])
def test_attention_refusals(parrot_lib, rows, msg, status):
    r = parrot.make_tree_rows(*rows)
    refused(plan(parrot_lib, rows=r), msg, status)
    refused(attend(parrot_lib, rows=r), msg, status)
    for size in (parrot.parrot_cache8_plan_bytes, parrot.parrot_cache8_workspace_bytes):
        with pytest.raises(B.ParrotError, match=msg.replace("^", r"\^")):
            size(problem(), r)


def test_attention_more_refusals(parrot_lib):
    rows = parrot.make_tree_rows(20, 10, 20, 8)
    need, ws = parrot.parrot_cache8_plan_bytes(problem(), rows), parrot.parrot_cache8_workspace_bytes(problem(), rows)
    assert need % 256 == 0 and need > 0 and ws > 0
    refused(plan(parrot_lib, size=need - 1), "plan is", B.PARROT_ERR_WORKSPACE_TOO_SMALL)
    refused(attend(parrot_lib, plan_bytes=need - 1), "plan is", B.PARROT_ERR_WORKSPACE_TOO_SMALL)
    refused(attend(parrot_lib, room=ws - 1), "workspace is", B.PARROT_ERR_WORKSPACE_TOO_SMALL)
    refused(attend(parrot_lib, prob=problem(num_requests=0)), "no requests")
    none = parrot.make_tree_rows(0, 0, 0, 8)
    assert plan(parrot_lib, rows=none, plan=None) == B.PARROT_OK and attend(parrot_lib, rows=none, q=None) == B.PARROT_OK
    assert parrot.parrot_cache8_plan_bytes(problem(), none) == 0 == parrot.parrot_cache8_workspace_bytes(problem(), none)


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("heads,ratio", [(4, 2), (40, 1), (1, 71), (7, 3)])
def test_sizes_never_decrease(parrot_lib, dtype, heads, ratio):
    """Growing any count or length, one after another, in steps over every tile width."""
    sizes = dict(num_requests=1, num_groups=0, max_prefix_len=16, max_suffix_len=1, max_prefix_depth=0, T=1, most=1, group=0)
    grow = dict(T=[2, 17, 64, 500], most=[2, 5, 16, 33, 300], max_suffix_len=[40, 300, 9000], num_requests=[2, 8, 300],
                num_groups=[1, 3, 60], max_prefix_len=[100, 3000], group=[1, 5, 40, 500], max_prefix_depth=[1, 2, 4])

    def size(s):
        prob = problem(num_heads=heads, dtype=dtype, num_requests=s["num_requests"], num_groups=s["num_groups"],
                       max_group_size=1, max_prefix_len=s["max_prefix_len"], max_suffix_len=s["max_suffix_len"],
                       prefix_table_stride=1000, suffix_table_stride=1000, max_prefix_depth=s["max_prefix_depth"])
        rows = parrot.make_tree_rows(s["T"], min(s["most"], s["max_suffix_len"]), min(s["group"], s["T"]), heads * ratio)
        return parrot.parrot_cache8_plan_bytes(prob, rows), parrot.parrot_cache8_workspace_bytes(prob, rows)

    for seed in range(6):
        rng = np.random.default_rng(seed)
        s, at = dict(sizes), {k: list(v) for k, v in grow.items()}
        was = size(s)
        while at:
            k = list(at)[int(rng.integers(0, len(at)))]
            s[k] = at[k].pop(0)
            if not at[k]:
                del at[k]
            now = size(s)
            assert now[0] >= was[0] and now[1] >= was[1], (seed, k, s)
            was = now


def test_copy_refusals(parrot_lib):
    def call(pools, n=3, blocks=10, src=FAKE, dst=FAKE + 4096, count=None):
        array = (B.ParrotBlockPool * max(len(pools), 1))(*(B.ParrotBlockPool(*p) for p in pools))
        return parrot_lib.parrot_copy_blocks(array, len(pools) if count is None else count, blocks, src, dst, n, None, None)
    good = [(FAKE + (1 << 20), 4096)]
    refused(call(good, n=-1), "num_copies")
    refused(call(good, blocks=0), "num_blocks")
    refused(call(good, count=-1), "num_pools")
    refused(call(good, src=None), "src is NULL")
    refused(call(good, dst=FAKE + 2), "dst is not")
    refused(call(good, src=FAKE, dst=FAKE), "same array")
    refused(call([(None, 4096)]), "pool 0 is NULL")
    refused(call(good + [(FAKE + 8, 4096)]), "pool 1 is not aligned")
    for n in (0, 3, -2, 1 << 40):
        refused(call(good + [(FAKE, n)]), "block_bytes of pool 1")
    assert call(good, n=0) == B.PARROT_OK and call([]) == B.PARROT_OK
    assert parrot_lib.parrot_copy_blocks(None, 1, 10, FAKE, FAKE + 4096, 3, None, None) == B.PARROT_ERR_INVALID_ARGUMENT


def test_python_forms_refuse_pools():
    p = problem(num_suffix_blocks=4)
    good = parrot.cache8_pools(4, 4, 128, device="cpu")
    from paper_2405_19888_amd.cache8 import _pool
    dev = torch.device("cpu")
    _pool(good, "suffix", 4, p, dev)
    with pytest.raises(ValueError, match="dict"):
        _pool([good["k"]], "suffix", 4, p, dev)
    for bad in (dict(good, k=good["k"][:3]), dict(good, v=good["v"].view(torch.uint8).flatten(2)),
                dict(good, scales=good["scales"].view(torch.uint8).short()),
                dict(good, k=good["k"].view(torch.uint8).transpose(2, 3))):
        with pytest.raises(ValueError, match="8-bit tensor"):
            _pool(bad, "suffix", 4, p, dev)
    with pytest.raises(ValueError, match="is on"):
        _pool(good, "suffix", 4, p, torch.device("cuda", 0))
    with pytest.raises(ValueError, match="head_dim"):
        parrot.cache8_pools(4, 4, 80, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        parrot.copy_blocks([good["k"]], [0], [1])


def test_values_of_pools():
    rng = np.random.default_rng(0)
    dense = [rng.normal(size=(3, 2, 16, 128)) * 2.0 ** rng.integers(-5, 5, (3, 2, 1, 1)) for _ in range(2)]
    packed = [oracle.pack(x) for x in dense]
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x))
    pools = {"k": t(packed[0][0]), "v": t(oracle.value_order(packed[1][0])), "scales": t(np.stack([packed[0][1], packed[1][1]], -1))}
    k, v = parrot.cache8_values(pools)
    assert np.array_equal(k.double().numpy(), oracle.values(*packed[0]))
    assert np.array_equal(v.double().numpy(), oracle.values(*packed[1]))
    k, v = parrot.cache8_values(pools, blocks=[2, 0])
    assert np.array_equal(v.double().numpy(), oracle.values(*packed[1])[[2, 0]])


# ------------------------------------------------------------- the oracle's pins
def test_codes_match_torch():
    codes = np.arange(256, dtype=np.uint8)
    values = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    got = oracle.decode(codes)
    assert np.array_equal(np.isnan(got), np.isnan(values)) and np.array_equal(got[~np.isnan(got)], values[~np.isnan(got)])
    rng = np.random.default_rng(0)
    x = np.clip(rng.normal(size=50000) * np.exp(4 * rng.normal(size=50000)), -448, 448).astype(np.float32)
    assert np.array_equal(oracle.encode(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert np.array_equal(oracle.encode(got[~np.isnan(got)]), codes[~np.isnan(got)])
    # ties go to the even code, half the least size to zero
    assert oracle.encode([17, 19, 2.0 ** -10, 3 * 2.0 ** -10]).tolist() == [88, 90, 0, 2]


def test_scales_by_hand():
    need = lambda x: int(oracle.need(np.array([[x]]), (0, 1)))
    assert [need(x) for x in (448.0, 448.1, 224.0, 224.1, 1.0, 0.875, 0.0)] == [127, 128, 126, 127, 119, 118, 0]
    assert need(1e-300) == 1 and oracle.scale(1) == 2.0 ** -126
    assert need(float("inf")) == 0


def test_orders_are_each_others_inverse():
    x = np.arange(16 * 128).reshape(1, 16, 128)
    y = oracle.value_order(x)
    assert y.shape == (1, 2, 4, 16, 4, 4) and np.array_equal(oracle.token_order(y), x)
    assert y[0, 1, 2, 5, 3, 1] == x[0, 4 * 2 + 1, 64 + 4 * 5 + 3]


def test_fill_by_hand():
    """One block of one head: a token of size 1 before, one of size 500 after it."""
    codes = np.zeros((1, 1, 16, 64), dtype=np.uint8)
    codes[0, 0, 0, 0], codes[0, 0, 0, 1] = oracle.encode([448.0])[0], oracle.encode([1.5 * 2.0 ** -6])[0]
    byte = np.array([[127 - 8]])               # scale 2^-8: the token is (1.75, 1.5 * 2^-14)
    new = np.zeros((1, 1, 64))
    new[0, 0, 3] = 500.0
    got, now = oracle.fill(new, codes, byte, [0, 1], [[0]], [2])
    assert now[0, 0] == 128                    # 2: 500 / 2 <= 448 < 500
    v = oracle.values(got, now)[0, 0]
    assert v[0, 0] == 1.75 and v[0, 1] == 0.0 and v[1, 3] == 512.0   # (250 is a tie between 240 and 256... codes step 16)
    again, byte2 = oracle.fill(new * 0, got, now, [0, 1], [[0]], [1])     # the first slot again: a new block
    assert byte2[0, 0] == 0 and not again[0, 0, 0].any()


def test_planted_mistakes_are_caught():
    """Rounding that is not to even, a scale one too small, and slots exchanged change the pins."""
    assert oracle.encode([17.0])[0] != oracle.encode([17.0001])[0]
    x = np.random.default_rng(1).normal(size=(2, 1, 16, 64))
    codes, byte = oracle.pack(x)
    assert np.abs(oracle.values(codes, byte) - x).max() <= 2.0 ** -4 * np.abs(x).max()
    assert np.abs(oracle.values(codes, byte + 1) - x).max() > 0.5
    assert not np.array_equal(oracle.value_order(codes).reshape(-1), codes.reshape(-1))
