"""A drafting step on the host: refusals before any device work, rotary embeddings,
the store's truncation, and pins of the oracle the GPU tests compare with."""
import ctypes
import math

import numpy as np
import pytest
import torch

import drafts_util as du
import paper_2405_19888_amd as parrot
from drafts_util import oracle
from oracle import shared_prefix_prefill
from paper_2405_19888_amd import binding as B
from paper_2405_19888_amd.context import ContextStore

FAKE = 1 << 20          # aligned fake device addresses: never dereferenced here


def problem(**over):
    kw = dict(num_requests=8, num_heads=4, head_dim=128, block_size=16, num_groups=2, max_group_size=8,
              max_prefix_len=500, max_suffix_len=300, prefix_table_stride=32, suffix_table_stride=19,
              num_prefix_blocks=100, num_suffix_blocks=100, dtype=1, sm_scale=0.1)
    kw.update(over)
    return B.make_problem(**kw)


def fill_rows(**over):
    kw = dict(num_query_rows=20, max_query_rows=10, num_query_heads=8, norm_eps=1e-6, q_stride=1024, k_stride=512,
              v_stride=512)
    kw.update(over)
    return B.ParrotFillRows(*kw.values())


def addresses(names, over):
    vals = {n: FAKE + 4096 * i for i, n in enumerate(names)}
    vals.update(over)
    return [vals[n] for n in names]


FILL = ["q", "k", "v", "q_norm", "k_norm", "positions", "query_offsets", "suffix_block_tables", "suffix_lens", "q_out",
        "suffix_k", "suffix_v"]
TREE = ["q", "query_offsets", "tree_parents", "prefix_k", "prefix_v", "suffix_k", "suffix_v", "prefix_block_tables",
        "prefix_lens", "prefix_parents", "suffix_block_tables", "suffix_lens", "group_ids", "out", "lse", "workspace"]
ACCEPT = ["query_offsets", "tree_parents", "draft_tokens", "target_tokens", "root_tokens", "accept_rows",
          "accept_lens", "next_tokens"]
COMMIT = ["query_offsets", "accept_rows", "accept_lens", "suffix_block_tables", "suffix_lens", "suffix_k", "suffix_v",
          "committed_lens"]


def call(lib, fn, prob=None, rows=None, rotary=None, requests=8, ws=1 << 45, **over):
    prob = problem() if prob is None else prob
    if fn == "parrot_rotary_fill":
        rows = fill_rows() if rows is None else rows
        return lib.parrot_rotary_fill(ctypes.byref(prob), ctypes.byref(rows), rotary, *addresses(FILL, over), None, None)
    rows = parrot.make_tree_rows(20, 10, 20, 8) if rows is None else rows
    if fn == "parrot_shared_prefix_tree_decode":
        return lib.parrot_shared_prefix_tree_decode(ctypes.byref(prob), ctypes.byref(rows), *addresses(TREE, over), ws,
                                                    None, None)
    if fn == "parrot_tree_accept":
        return lib.parrot_tree_accept(requests, ctypes.byref(rows), *addresses(ACCEPT, over), None, None)
    return lib.parrot_tree_commit(ctypes.byref(prob), ctypes.byref(rows), *addresses(COMMIT, over), None, None)


def test_struct_layouts():
    assert ctypes.sizeof(B.ParrotRotary) == 16 + 64 * 8
    assert ctypes.sizeof(B.ParrotRotaryConfig) == 8 + 8 + 8 + 5 * 8
    assert ctypes.sizeof(B.ParrotFillRows) == 4 * 4 + 3 * 8
    assert ctypes.sizeof(B.ParrotTreeRows) == 4 * 4


@pytest.mark.parametrize("fn,names,optional", [
    ("parrot_rotary_fill", FILL, {"q_norm", "k_norm", "positions"}),
    ("parrot_shared_prefix_tree_decode", TREE, {"tree_parents", "prefix_parents"}),
    ("parrot_tree_accept", ACCEPT, {"tree_parents"}),
    ("parrot_tree_commit", COMMIT, set())])
def test_pointers(parrot_lib, fn, names, optional):
    """Every pointer is refused when NULL (but for the optional ones) or misaligned."""
    for n in names:
        if n not in optional:
            assert call(parrot_lib, fn, **{n: None}) == B.PARROT_ERR_INVALID_ARGUMENT, n
            assert "NULL" in B.parrot_last_error(), n
        if n != "positions":             # (unused without a rotation)
            assert call(parrot_lib, fn, **{n: FAKE + 1}) == B.PARROT_ERR_INVALID_ARGUMENT, n
            assert "aligned" in B.parrot_last_error(), n
    rot = ctypes.byref(parrot.make_rotary(64))
    if fn == "parrot_rotary_fill":
        for bad in (None, FAKE + 2):
            assert call(parrot_lib, fn, rotary=rot, positions=bad) == B.PARROT_ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("over,msg", [
    (dict(num_query_rows=-1), "num_query_rows"), (dict(max_query_rows=0), "max_query_rows"),
    (dict(max_query_rows=301), "max_query_rows"), (dict(num_query_heads=0), "num_query_heads"),
    (dict(norm_eps=-1.0), "norm_eps"), (dict(norm_eps=float("nan")), "norm_eps"),
    (dict(q_stride=1016), "q_stride"), (dict(k_stride=516), "16 bytes"), (dict(v_stride=-512), "v_stride"),
    (dict(q_stride=1 << 41), "q_stride")])
def test_fill_refusals(parrot_lib, over, msg):
    assert call(parrot_lib, "parrot_rotary_fill", rows=fill_rows(**over)) == B.PARROT_ERR_INVALID_ARGUMENT
    assert msg in B.parrot_last_error()


def test_fill_more_refusals(parrot_lib):
    wide = ctypes.byref(parrot.make_rotary(128))
    assert call(parrot_lib, "parrot_rotary_fill", prob=problem(head_dim=64), rotary=wide) == B.PARROT_ERR_INVALID_ARGUMENT
    assert "head_dim" in B.parrot_last_error()
    broken = parrot.make_rotary(64)
    broken.rotary_dim = 63
    assert call(parrot_lib, "parrot_rotary_fill", rotary=ctypes.byref(broken)) == B.PARROT_ERR_INVALID_ARGUMENT
    assert call(parrot_lib, "parrot_rotary_fill", rows=fill_rows(q_stride=2048), q=FAKE, q_out=FAKE) == \
        B.PARROT_ERR_INVALID_ARGUMENT
    assert "q_out" in B.parrot_last_error()
    assert call(parrot_lib, "parrot_rotary_fill", prob=problem(head_dim=80)) == B.PARROT_ERR_UNSUPPORTED
    assert call(parrot_lib, "parrot_rotary_fill", prob=problem(num_requests=0)) == B.PARROT_ERR_INVALID_ARGUMENT
    assert call(parrot_lib, "parrot_rotary_fill", rows=fill_rows(num_query_rows=0), k=None) == B.PARROT_OK


@pytest.mark.parametrize("rows,msg,status", [
    ((-1, 10, 20, 8), "num_query_rows", 1), ((20, 0, 20, 8), "max_query_rows", 1), ((20, 129, 20, 8), "128", 1),
    ((20, 10, 21, 8), "max_group_rows", 1), ((20, 10, -1, 8), "max_group_rows", 1), ((20, 10, 20, 6), "multiple", 1),
    ((20, 10, 20, 0), "multiple", 1), ((1 << 30, 128, 20, 8), "2^31", 2)])
def test_tree_refusals(parrot_lib, rows, msg, status):
    r = parrot.make_tree_rows(*rows)
    assert call(parrot_lib, "parrot_shared_prefix_tree_decode", rows=r) == status
    assert msg in B.parrot_last_error()
    with pytest.raises(B.ParrotError, match=msg.replace("^", r"\^")):
        parrot.parrot_tree_workspace_bytes(problem(), r)


def test_tree_more_refusals(parrot_lib):
    fn = "parrot_shared_prefix_tree_decode"
    assert call(parrot_lib, fn, prob=problem(max_suffix_len=9, suffix_table_stride=1)) == B.PARROT_ERR_INVALID_ARGUMENT
    assert call(parrot_lib, fn, prob=problem(sm_scale=float("inf"))) == B.PARROT_ERR_INVALID_ARGUMENT
    assert call(parrot_lib, fn, rows=parrot.make_tree_rows(0, 0, 0, 0), q=None) == B.PARROT_OK
    need = parrot.parrot_tree_workspace_bytes(problem(), parrot.make_tree_rows(20, 10, 20, 8))
    if need:
        assert call(parrot_lib, fn, ws=need - 1) == B.PARROT_ERR_WORKSPACE_TOO_SMALL


def test_tree_path_by_size(parrot_lib):
    """Short calls take one launch and no workspace to speak of, few long requests and
    prefixes of many rows the split plan; a nested problem's flat calls the same one."""
    def split(prob, rows, nested):
        return parrot_lib.parrot_test_tree_split(ctypes.byref(prob), ctypes.byref(rows), nested)

    def of(**over):
        return problem(num_groups=0, max_group_size=0, max_prefix_len=0, num_prefix_blocks=0, **over)

    few = parrot.make_tree_rows(32, 8, 0, 8)
    short, long = of(), of(max_suffix_len=30000, suffix_table_stride=1875)
    assert split(short, few, 0) == 0 and split(long, few, 0) == 1
    assert parrot.parrot_tree_workspace_bytes(short, few) == 256
    assert parrot.parrot_tree_workspace_bytes(long, few) > 32 * 8 * 128 * 4
    many = parrot.make_tree_rows(2000, 32, 1000, 8)
    shared = problem(num_requests=64, max_group_size=32, max_prefix_len=4096, prefix_table_stride=256, max_prefix_depth=2)
    assert split(shared, many, 0) == split(shared, many, 1) == 1


def drawn_sizes(rng):
    """Sizes of a tree call: [requests, groups, prefix, own tokens, depth, rows, most, group rows]."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    R, most, own = log(1, 300), log(1, 128), log(128, 40000)
    T = int(rng.integers(1, R * most + 1))
    return [R, int(rng.integers(0, 12)), log(1, 100000), own, int(rng.integers(0, 5)), T, most, int(rng.integers(0, T + 1))]


def tree_sizes(sizes, heads, ratio, dim, dtype):
    R, ng, pre, own, depth, T, most, group = sizes
    prob = problem(num_requests=R, num_heads=heads, head_dim=dim, num_groups=ng, max_group_size=min(R, 1 if ng else 0),
                   max_prefix_len=pre if ng else 0, max_suffix_len=own, prefix_table_stride=-(-pre // 16),
                   suffix_table_stride=-(-own // 16), max_prefix_depth=depth, dtype=dtype)
    return prob, parrot.make_tree_rows(T, most, group if ng else 0, heads * ratio)


@pytest.mark.parametrize("heads,ratio", [(8, 4), (32, 1), (1, 8), (5, 3), (300, 1), (700, 1)])
@pytest.mark.parametrize("dim,dtype", [(128, 1), (64, 2), (128, 0), (64, 0)])
def test_tree_workspace_never_decreases(parrot_lib, heads, ratio, dim, dtype):
    """One workspace for the largest call serves every smaller one, whichever plan each takes."""
    used = parrot_lib.parrot_test_tree_used_bytes
    used.restype = ctypes.c_size_t
    rng = np.random.default_rng(heads * dim + dtype)
    changes = 0
    for _ in range(300):
        big = drawn_sizes(rng)
        prob, rows = tree_sizes(big, heads, ratio, dim, dtype)
        most = parrot.parrot_tree_workspace_bytes(prob, rows)
        for nested in (0, 1):
            assert used(ctypes.byref(prob), ctypes.byref(rows), nested) <= most
        for _ in range(8):
            small = [x if rng.random() < 0.4 else int(rng.integers(min(x, i not in (1, 4, 7)), x + 1)) for i, x in enumerate(big)]
            small[3], small[7] = max(small[3], small[6]), min(small[7], small[5])
            if small[3] > big[3]:
                continue
            prob, rows = tree_sizes(small, heads, ratio, dim, dtype)
            less = parrot.parrot_tree_workspace_bytes(prob, rows)
            assert less <= most, (big, small)
            changes += used(ctypes.byref(prob), ctypes.byref(rows), 0) > 0
    assert changes > 100                          # many of them take the split plan


@pytest.mark.parametrize("levels", [0, 1, 2, 3, 4])
def test_join_stays_inside_a_row(parrot_lib, levels):
    """The join's slots: chunks of every level and pieces where they stand, and inside the
    row's slots whatever a descriptor that nobody wrote holds."""
    rng = np.random.default_rng(levels)
    out = (ctypes.c_int * 4096)()
    slots = lambda *a: out[:parrot_lib.parrot_test_tree_slots(*a, out, len(out))]
    for _ in range(200):
        chunks = int(rng.integers(1, 9)) if levels else 0
        before, pieces = levels * chunks, int(rng.integers(1, 9))
        seg = before + pieces
        n = [int(x) for x in rng.integers(0, chunks + 1, levels)]
        own = int(rng.integers(0, pieces + 1))
        want = [l * chunks + c for l in range(levels) for c in range(n[l])] + [before + i for i in range(own)]
        n += [0] * (4 - levels)
        assert slots(n[0] | n[1] << 16, n[2] | n[3] << 16, own, chunks, before, seg) == want
        for lo, hi, some in ((0xFFFFFFFF, 0xFFFFFFFF, 1 << 30), (0x00010001, 0x7FFF0003, -5),
                             *[(int(a), int(b), int(c)) for a, b, c in rng.integers(0, 1 << 31, (5, 3))]):
            got = slots(lo, hi, some, chunks, before, seg)
            assert len(got) <= seg and all(0 <= x < seg for x in got), (lo, hi, some, chunks, before, seg)


@pytest.mark.timeout(20)
def test_row_counts_of_bad_groups(parrot_lib):
    """Parents in a ring and group ids out of range, which the content check refuses, neither
    hang nor break the row counts on the host."""
    rows = parrot.tree_rows_from_host([0, 3, 5, 9], [1, 0, 7], 2, 8, prefix_parents=[1, 0])
    assert (rows.num_query_rows, rows.max_query_rows, rows.max_group_rows) == (9, 4, 5)
    rows = parrot.tree_rows_from_host([0, 3, 5], [1, 0], 2, 8, prefix_parents=[5, 0])
    assert rows.max_group_rows == 5


def tensors(dtype=torch.float16):
    """A tree and fill call's tensors for problem() with 20 rows of 8 query heads."""
    ints = lambda *n: torch.zeros(n, dtype=torch.int32)
    pool = torch.zeros((100, 4, 16, 128), dtype=dtype)
    return dict(q=torch.zeros((20, 8, 128), dtype=dtype), query_offsets=ints(9), tree_parents=ints(20), prefix_k=pool,
                prefix_v=pool, suffix_k=pool, suffix_v=pool, prefix_block_tables=ints(2, 32), prefix_lens=ints(2),
                prefix_parents=None, suffix_block_tables=ints(8, 19), suffix_lens=ints(8), group_ids=ints(8),
                out=torch.zeros((20, 8, 128), dtype=dtype), lse=torch.zeros((20, 8)),
                workspace=torch.zeros(256, dtype=torch.uint8))


@pytest.mark.parametrize("name", ["q", "query_offsets", "tree_parents", "prefix_k", "suffix_v", "prefix_block_tables",
                                  "prefix_lens", "suffix_block_tables", "suffix_lens", "group_ids", "out", "lse"])
def test_tensors_that_do_not_fit(parrot_lib, name):
    """A tensor of another type, too short or with gaps is refused by its name before the
    library sees its address; fitting ones get as far as the device check."""
    rows = parrot.make_tree_rows(20, 10, 20, 8)
    with pytest.raises(ValueError, match="on the GPU"):
        parrot.parrot_shared_prefix_tree_decode(problem(), rows, **tensors())
    x = tensors()[name]
    bads = [x.double()]
    if name != "tree_parents":                    # (padding rows' parents are not read)
        bads.append(x[:-1].clone())
    if x.shape[0] > 1:
        bads.append(torch.cat([x, x])[::2])
    for bad in bads:
        with pytest.raises(ValueError, match=name.replace("_block", "") + " is not a contiguous"):
            parrot.parrot_shared_prefix_tree_decode(problem(), rows, **{**tensors(), name: bad})


def test_workspace_and_checked_tensors_that_do_not_fit(parrot_lib):
    """A workspace with gaps or on another device, and every array and the scratch of the
    content check, are refused by name."""
    rows = parrot.make_tree_rows(20, 10, 20, 8)
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(512, dtype=torch.uint8)[::2],
                torch.zeros((16, 32)).t()):
        with pytest.raises(ValueError, match="workspace is not a contiguous"):
            parrot.parrot_shared_prefix_tree_decode(problem(), rows, **{**tensors(), "workspace": bad})
    with pytest.raises(ValueError, match="workspace is on meta"):
        parrot.parrot_shared_prefix_tree_decode(
            problem(), rows, **{**tensors(), "workspace": torch.zeros(512, dtype=torch.uint8, device="meta")})
    names = ["query_offsets", "tree_parents", "prefix_block_tables", "prefix_lens", "prefix_parents",
             "suffix_block_tables", "suffix_lens", "group_ids"]
    good = {n: tensors()[n] for n in names}
    good.update(prefix_parents=torch.zeros(2, dtype=torch.int32), scratch=torch.zeros(16, dtype=torch.int32))
    with pytest.raises(ValueError, match="on the GPU"):
        parrot.parrot_validate_tree_inputs(problem(), rows, **good)
    for name, x in good.items():
        bads = [x.long(), torch.cat([x, x])[::2]] + ([x[:-1].clone()] if name != "tree_parents" else [])
        for bad in bads:
            with pytest.raises(ValueError, match=name.replace("_block", "") + " is not a contiguous"):
                parrot.parrot_validate_tree_inputs(problem(), rows, **{**good, name: bad})


def test_parents_shorter_than_the_rows(parrot_lib, monkeypatch):
    """The library is told of no row whose parent the tensor does not hold."""
    from paper_2405_19888_amd import drafts
    told = []
    monkeypatch.setattr(drafts, "_bound", lambda fn, values, *_: lambda *_: told.append(values[1]._obj))
    monkeypatch.setattr(drafts, "_device", lambda t: t.device)
    counts = parrot.make_tree_rows(20, 10, 18, 8)
    t, ints = tensors(), [torch.zeros(n, dtype=torch.int32) for n in (20, 20, 8, 20, 8, 8)]
    for n in (25, 20, 19, 12, 0):
        parents = torch.full((n,), -1, dtype=torch.int32)
        parrot.parrot_shared_prefix_tree_decode(problem(), counts, **{**t, "tree_parents": parents})
        parrot.parrot_tree_accept(8, counts, t["query_offsets"], parents, *ints)
        for rows in told[-2:]:
            assert (rows.num_query_rows, rows.max_query_rows, rows.num_query_heads) == (min(n, 20), 10, 8)
            assert rows.max_group_rows == min(n, 18)
    parrot.parrot_shared_prefix_tree_decode(problem(), counts, **{**t, "tree_parents": None})
    assert told[-1].num_query_rows == 20 and counts.num_query_rows == 20 and counts.max_group_rows == 18


def test_fill_tensors_that_do_not_fit(parrot_lib):
    t = tensors()
    kv = torch.zeros((20, 4, 128), dtype=torch.float16)
    good = dict(q=t["q"], k=kv, v=kv, q_norm=None, k_norm=kv[0, 0], positions=t["tree_parents"],
                query_offsets=t["query_offsets"], suffix_tables=t["suffix_block_tables"], suffix_lens=t["suffix_lens"],
                q_out=t["out"], suffix_k=t["suffix_k"], suffix_v=t["suffix_v"])
    with pytest.raises(ValueError, match="on the GPU"):
        parrot.parrot_rotary_fill(problem(), 20, 10, 8, None, **good)
    for name, bad, msg in [("q", t["q"][:19], "q is not"), ("k", kv.float(), "k is not"), ("v", kv[:, :3], "v is not"),
                           ("k_norm", kv[0, 0, :64], "k_norm is not"), ("positions", t["tree_parents"].long(), "positions"),
                           ("q_out", t["out"][:10], "q_out is not"), ("suffix_k", t["suffix_k"][:99], "suffix_k is not")]:
        with pytest.raises(ValueError, match=msg):
            parrot.parrot_rotary_fill(problem(), 20, 10, 8, None, **{**good, name: bad})


def test_accept_and_commit_refusals(parrot_lib):
    assert call(parrot_lib, "parrot_tree_accept", requests=-1) == B.PARROT_ERR_INVALID_ARGUMENT
    assert call(parrot_lib, "parrot_tree_accept", requests=0, query_offsets=None,
                rows=parrot.make_tree_rows(0, 0, 0, 0)) == B.PARROT_OK
    assert call(parrot_lib, "parrot_tree_accept", requests=0) == B.PARROT_ERR_INVALID_ARGUMENT   # rows without requests
    assert call(parrot_lib, "parrot_tree_accept", accept_rows=FAKE, tree_parents=FAKE) == B.PARROT_ERR_INVALID_ARGUMENT
    for other in ("suffix_lens", "accept_lens"):
        assert call(parrot_lib, "parrot_tree_commit", committed_lens=FAKE, **{other: FAKE}) == \
            B.PARROT_ERR_INVALID_ARGUMENT
        assert "committed_lens" in B.parrot_last_error()
    assert call(parrot_lib, "parrot_tree_commit", suffix_k=FAKE, suffix_v=FAKE) == B.PARROT_ERR_INVALID_ARGUMENT
    assert call(parrot_lib, "parrot_tree_commit", prob=problem(num_suffix_blocks=1 << 28)) == B.PARROT_ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        parrot.tree_accept(torch.zeros(2, dtype=torch.int32), None, *[torch.zeros(1, dtype=torch.int32)] * 3)


# ------------------------------------------------------------ rotary embeddings
@pytest.mark.parametrize("scaling,kw", [("none", {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
                                        ("yarn", dict(factor=16.0, original_length=4096)),
                                        ("wavelength", dict(factor=8.0, original_length=8192)),
                                        ("wavelength", dict(factor=2.0, original_length=512, low=0.5, high=3.0))])
@pytest.mark.parametrize("rd,base", [(128, 10000.0), (64, 500000.0), (20, 10000.0)])
def test_rotary_frequencies(parrot_lib, scaling, kw, rd, base):
    rot = parrot.make_rotary(rd, base=base, scaling=scaling, **kw)
    radians, amplitude = oracle.rotary_frequencies(rd, base, scaling, **kw)
    assert rot.rotary_dim == rd and rot.amplitude == np.float32(amplitude)
    for i, f in enumerate(radians):
        # pow and the division by 2 pi: a few steps of 2^-53
        assert abs(rot.turns[i] / 2.0 ** 64 - f / (2 * math.pi)) <= 16 * 2.0 ** -53 * f / (2 * math.pi) + 2.0 ** -64
    same = parrot.rotary_from_frequencies(radians, amplitude=amplitude)
    assert all(abs(same.turns[i] - rot.turns[i]) <= 16 * 2.0 ** -53 * rot.turns[i] + 1 for i in range(rd // 2))


@pytest.mark.parametrize("rd,base", [(128, 10000.0), (64, 500000.0), (20, 7.5)])
@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 8.0)])
def test_rotary_turns_hold_at_far_positions(parrot_lib, rd, base, scaling, factor):
    """The stored fraction of a turn is the exact one's to 1.5 * 2^-64, so 2^31 positions keep
    the angle to 2^-32 turns (and its lower 32 bits, cut off, are another 2^-32)."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    exact = Decimal(base)
    if scaling == "ntk":
        exact *= Decimal(factor) ** (Decimal(rd) / (rd - 2))
    rot = parrot.make_rotary(rd, base=base, scaling=scaling, factor=factor)
    for i in range(rd // 2):
        f = exact ** (Decimal(-2 * i) / rd) / (Decimal(factor) if scaling == "linear" else 1)
        assert abs(Decimal(rot.turns[i]) - f / (2 * pi) * 2 ** 64) <= Decimal("1.5"), i
    for f in (0.0, 1.0, 0.1, 6.283185307179586, 2.0 ** -60):
        turns = parrot.rotary_from_frequencies([f]).turns[0]
        assert abs(Decimal(turns) - Decimal(f) / (2 * pi) * 2 ** 64) <= Decimal("1.5"), f


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=130), dict(base=1.0), dict(base=float("nan")),
    dict(scaling="linear", factor=0.5), dict(scaling="yarn", factor=4.0), dict(scaling="ntk", rotary_dim=2, factor=2.0),
    dict(scaling="yarn", factor=float("inf"), original_length=4096), dict(amplitude=-1.0),
    dict(scaling="wavelength", factor=2.0, original_length=100, low=4.0, high=1.0), dict(amplitude=1e39)])
def test_rotary_refusals(parrot_lib, kw):
    with pytest.raises(B.ParrotError):
        parrot.make_rotary(**{"rotary_dim": 64, **kw})


def test_amplitude_that_is_no_positive_float(parrot_lib):
    """An amplitude below the least float would scale every rotated pair by zero."""
    for bad in (1e-50, 5e-324):
        with pytest.raises(B.ParrotError, match="amplitude"):
            parrot.make_rotary(64, amplitude=bad)
        with pytest.raises(B.ParrotError, match="amplitude"):
            parrot.rotary_from_frequencies([0.1], amplitude=bad)
    assert parrot.make_rotary(64, amplitude=2.0 ** -149).amplitude == 2.0 ** -149


def test_rotary_from_frequencies_refusals(parrot_lib):
    for bad in ([-0.1], [7.0], [float("nan")], [0.1] * 65, []):
        with pytest.raises(B.ParrotError):
            parrot.rotary_from_frequencies(bad)
    with pytest.raises(ValueError):
        parrot.make_rotary(64, scaling="unknown")


# -------------------------------------------------------------------- the store
def test_truncate(parrot_lib):
    st = ContextStore(16, 10)
    c = st.fill(list(range(20)), [16])
    for _ in range(30):
        st.append(c)
    assert st.own_tokens(c) == 34 and st.free_blocks == 10 - 1 - 3
    st.truncate(c, 33)
    assert st.free_blocks == 6 and st.own_tokens(c) == 33
    st.truncate(c, 32)
    assert st.free_blocks == 7
    st.append(c)                                         # a new block again
    assert st.free_blocks == 6 and st.own_tokens(c) == 33
    table = st.build_batch([c]).suffix_tables[0].copy()
    st.truncate(c, 20)
    st.append(c)
    assert np.array_equal(st.build_batch([c]).suffix_tables[0][:2], table[:2]) and st.own_tokens(c) == 21
    for bad in (-1, 22):
        with pytest.raises(B.ParrotError):
            st.truncate(c, bad)
    with pytest.raises(B.ParrotError):
        st.truncate(c + 1, 0)
    st.truncate(c, 0)
    assert st.free_blocks == 9
    st.free(c)
    assert st.free_blocks == 10


# ------------------------------------------------------------------ oracle pins
def small_tree(parents, heads=2, ratio=2, dim=64, cached=5):
    rows = [len(parents)]
    plan = du.tree_plan("float32", heads, dim, [0], [7], [cached], rows, seed=1)
    batch = du.make_batch(plan, seed=2)
    return plan, batch, du.queries(rows[0], heads * ratio, dim, "float32")


def tree_oracle(plan, batch, q, parents, **over):
    kw = dict(sm_scale=plan.sm_scale)
    kw.update(over)
    return oracle.shared_prefix_tree(q, [0, q.shape[0]], parents, batch.k_pool, batch.v_pool, batch.k_pool,
                                     batch.v_pool, plan.prefix_tables, plan.prefix_lens, plan.suffix_tables,
                                     plan.suffix_lens, plan.group_ids, **kw)


def test_tree_oracle_against_masked_attention():
    parents = np.array([-1, 0, 0, 1, -1, 3])
    plan, batch, q = small_tree(parents)
    out, lse, _, _ = tree_oracle(plan, batch, q, parents)
    seen = {0: [0], 1: [0, 1], 2: [0, 2], 3: [0, 1, 3], 4: [4], 5: [0, 1, 3, 5]}        # by hand
    mask = torch.zeros(6, 18, dtype=torch.bool)
    mask[:, :12] = True
    for j, s in seen.items():
        mask[j, [12 + a for a in s]] = True
    from oracle import request_kv
    K, V = request_kv(0, prefix_k=batch.k_pool, prefix_v=batch.v_pool, suffix_k=batch.k_pool, suffix_v=batch.v_pool,
                      prefix_tables=plan.prefix_tables, prefix_lens=plan.prefix_lens, suffix_tables=plan.suffix_tables,
                      suffix_lens=plan.suffix_lens, group_ids=plan.group_ids)
    k, v = (torch.from_numpy(x).transpose(0, 1).repeat_interleave(2, 0) for x in (K, V))
    want = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1), k, v, attn_mask=mask,
                                                            scale=plan.sm_scale).transpose(0, 1)
    assert np.abs(out - want.numpy()).max() <= 1e-12


def test_tree_oracle_chain_is_prefill():
    plan, batch, q = small_tree([-1, 0, 1, 2], ratio=1)
    for parents in (None, [-1, 0, 1, 2]):
        out, lse, _, _ = tree_oracle(plan, batch, q, parents)
        pout, plse = shared_prefix_prefill(q, [0, 4], batch.k_pool, batch.v_pool, batch.k_pool, batch.v_pool,
                                           plan.prefix_tables, plan.prefix_lens, plan.suffix_tables, plan.suffix_lens,
                                           plan.group_ids, plan.sm_scale)
        assert np.abs(out - pout).max() <= 1e-12 and np.abs(lse - plse).max() <= 1e-12


def test_rotate_keeps_lengths_and_relative_angles():
    """A rotation keeps each pair's length, and the product of a query and a key depends
    on the difference of their positions alone."""
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(1, 1, 64)), rng.normal(size=(1, 1, 64))
    f, a = oracle.rotary_frequencies(64)
    for inter in (False, True):
        turn = lambda x, p: oracle.rotate(x, [p], f, inter, a)[0]
        assert abs((turn(q, 77) ** 2).sum() - (q ** 2).sum()) <= 1e-10
        assert abs((turn(q, 5) * turn(k, 2)).sum() - (turn(q, 1003) * turn(k, 1000)).sum()) <= 1e-9
        assert np.abs(turn(q, 0) - q).max() == 0
    # pair (1, 0) at a quarter turn becomes (0, 1)
    x = np.zeros((1, 1, 4))
    x[0, 0, 0] = 1
    y = oracle.rotate(x, [1], [math.pi / 2, 0.0], False, 1.0)[0][0, 0]
    assert np.allclose(y, [0, 0, 1, 0], atol=1e-15)


def test_accept_oracle_by_hand():
    # rows 0 and 1 start; 2 and 3 follow 0; 4 follows 3; tokens 9 from the root, 5 after row 0, 6 after row 3
    up, draft, target = [-1, -1, 0, 0, 3], [9, 9, 4, 5, 6], [5, 0, 0, 6, 8]
    rows, lens, follow = oracle.tree_accept([0, 5], up, draft, target, [9])
    assert list(rows) == [0, 3, 4, -1, -1] and lens[0] == 3 and follow[0] == 8


def test_commit_oracle_by_hand():
    moves, after = oracle.tree_commit([0, 4], [0, 2, 3, -1], [3], [[7, 3]], [18])
    assert moves == [((7, 14), (7, 14)), ((3, 0), (7, 15)), ((3, 1), (3, 0))] and after[0] == 17
