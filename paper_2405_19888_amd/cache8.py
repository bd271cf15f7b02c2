"""Caches held in 8 bits, and copies of cache blocks, through libparrot_attn (argument
marshalling only): fill of new rows, attention of single tokens, drafted chains and prompts,
blocks copied for forked contexts or moved together.

The ``parrot_*`` functions forward to the C entry points of the same name in
``include/parrot_attn.h``, which has the format; ``Cache8Filler``, ``Cache8Planner``,
``Cache8Decoder`` and ``BlockCopier`` keep the buffers of one batch shape and bind a call once;
``cache8_fill``, ``cache8_attention`` and ``copy_blocks`` are one-call forms on torch tensors.

A layer's pools are a dict of ``k`` (float8_e4m3fn [blocks, H, 16, D]), ``v`` (float8_e4m3fn
[blocks, H, D / 64, 4, 16, 4, 4]) and ``scales`` (float8_e8m0fnu [blocks, H, 2]); bytes (uint8) of
the same shapes do as well.  ``cache8_pools`` makes them, ``cache8_values`` reads them.

A step of an engine: per layer a ``Cache8Filler`` with the new rows' projections; a
``Cache8Planner`` once, as lengths and groups are the same in every layer, then a
``Cache8Decoder`` per layer.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from .binding import (PARROT_ERR_INVALID_ARGUMENT, ParrotBlockPool, ParrotCache8, ParrotError, ParrotFillRows,
                      ParrotProblem, ParrotRotary, ParrotTreeRows, _check, _on_stream, _ptr, _sizes_from_tensors,
                      load_library, make_problem, parrot_last_error)
from .drafts import (_TORCH_DTYPES, _bound, _device, _most_rows, _need, _need_rows, _need_tree, _row_stride, _stream,
                     tree_rows_from_host)

_CODES = (torch.float8_e4m3fn, torch.uint8)
_SCALES = (torch.float8_e8m0fnu, torch.uint8)


# -------------------------------------------------------------------- the pools
def cache8_pools(num_blocks: int, heads: int, head_dim: int, device="cuda") -> dict:
    """The pools of one layer, all zeros."""
    if head_dim not in (64, 128):
        raise ValueError(f"head_dim {head_dim} is not 64 or 128")
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)
    return {"k": zeros(num_blocks, heads, 16, head_dim).view(torch.float8_e4m3fn),
            "v": zeros(num_blocks, heads, head_dim // 64, 4, 16, 4, 4).view(torch.float8_e4m3fn),
            "scales": zeros(num_blocks, heads, 2).view(torch.float8_e8m0fnu)}


def cache8_values(pools: dict, blocks=None):
    """(keys, values) float32 [blocks, H, 16, D] that the pools stand for, of all blocks or of
    those listed (a look at the cache, not a path of it)."""
    k, v, s = (pools[x].view(torch.uint8) for x in ("k", "v", "scales"))
    if blocks is not None:
        k, v, s = k[blocks], v[blocks], s[blocks]
    as_float = lambda x: x.contiguous().view(torch.float8_e4m3fn).float()
    v = as_float(v).permute(0, 1, 3, 6, 2, 4, 5).reshape(k.shape)          # x g c d t -> (g t) (x c d)
    power = (s.int() - 127)[..., None, None]
    return torch.ldexp(as_float(k), power[:, :, 0]), torch.ldexp(v, power[:, :, 1])


def _shapes(blocks: int, heads: int, dim: int) -> dict:
    return {"k": (blocks, heads, 16, dim), "v": (blocks, heads, dim // 64, 4, 16, 4, 4), "scales": (blocks, heads, 2)}


def _pool(pools, name: str, blocks: int, p: ParrotProblem, device: torch.device) -> ParrotCache8:
    """The C struct of a layer's pools; refuses tensors that the kernels would leave."""
    if not isinstance(pools, dict) or any(x not in pools for x in ("k", "v", "scales")):
        raise ValueError(f"{name} is not a dict of k, v and scales")
    for x, (n, *rest) in _shapes(blocks, p.num_heads, p.head_dim).items():
        t = pools[x]
        if not isinstance(t, torch.Tensor):
            continue
        if t.dtype not in (_SCALES if x == "scales" else _CODES) or not t.is_contiguous() or t.dim() != len(rest) + 1 or \
                list(t.shape[1:]) != rest or t.shape[0] < n:
            raise ValueError(f"{name}[{x!r}] is not a contiguous 8-bit tensor of at least {[n, *rest]}")
        if t.device != device:
            raise ValueError(f"{name}[{x!r}] is on {t.device}, not on {device}")
    return ParrotCache8(*(_ptr(pools[x]) for x in ("k", "v", "scales")))


def parrot_cache8_plan_bytes(problem: ParrotProblem, rows: ParrotTreeRows) -> int:
    return _size("parrot_cache8_plan_bytes", problem, rows)


def parrot_cache8_workspace_bytes(problem: ParrotProblem, rows: ParrotTreeRows) -> int:
    return _size("parrot_cache8_workspace_bytes", problem, rows)


def _size(fn: str, problem, rows) -> int:
    n = getattr(load_library(), fn)(ctypes.byref(problem), ctypes.byref(rows))
    if n == ctypes.c_size_t(-1).value:
        raise ParrotError(PARROT_ERR_INVALID_ARGUMENT, parrot_last_error())
    return int(n)


# ---------------------------------------------------------------- marshalling
def _fill_call(problem, num_query_rows, max_query_rows, num_query_heads, rotary, norm_eps, q, k, v, q_norm, k_norm,
               positions, query_offsets, suffix_tables, suffix_lens, q_out, suffix, stream):
    T, D, dt, R = int(num_query_rows), problem.head_dim, _TORCH_DTYPES[problem.dtype], problem.num_requests
    for x, name, heads in ((q, "q", int(num_query_heads)), (k, "k", problem.num_heads), (v, "v", problem.num_heads)):
        _need_rows(x, name, T, heads, problem, k.device)
    _need(q_out, "q_out", dt, T * int(num_query_heads) * D, k.device)
    for x, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        _need(x, name, dt, D, k.device)
    for x, name, least in ((positions, "positions", T), (query_offsets, "query_offsets", R + 1),
                           (suffix_tables, "suffix_tables", R * problem.suffix_table_stride),
                           (suffix_lens, "suffix_lens", R)):
        _need(x, name, torch.int32, least, k.device)
    pool = _pool(suffix, "suffix", problem.num_suffix_blocks, problem, k.device)
    rows = ParrotFillRows(T, int(max_query_rows), int(num_query_heads), float(norm_eps),
                          0 if q is None else _row_stride(q, "q"), _row_stride(k, "k"), _row_stride(v, "v"))
    call = _bound(load_library().parrot_cache8_fill,
                  (ctypes.byref(problem), ctypes.byref(rows), None if rotary is None else ctypes.byref(rotary), q, k, v,
                   q_norm, k_norm, positions, query_offsets, suffix_tables, suffix_lens, q_out, ctypes.byref(pool)),
                  _device(k), stream)
    call.pools = suffix                          # (the struct holds addresses only)
    return call


def parrot_cache8_fill(problem, num_query_rows, max_query_rows, num_query_heads, rotary, q, k, v, q_norm, k_norm,
                       positions, query_offsets, suffix_tables, suffix_lens, q_out, suffix, norm_eps=0.0, stream=None,
                       trace=None):
    """Norm, rotate and cache new rows in 8 bits (see the C header).  The row strides come
    from q, k and v ([rows, heads, D], heads adjacent); q and q_out may be None."""
    _fill_call(problem, num_query_rows, max_query_rows, num_query_heads, rotary, norm_eps, q, k, v, q_norm, k_norm,
               positions, query_offsets, suffix_tables, suffix_lens, q_out, suffix, stream)(trace)


def _plan_call(problem, rows, query_offsets, prefix_lens, prefix_parents, suffix_lens, group_ids, plan, stream):
    p, device = problem, query_offsets.device
    _need_tree(p, device, query_offsets, None, None, prefix_lens, prefix_parents, None, suffix_lens, group_ids)
    _need(plan, "plan", torch.int32, 0, device)            # (its size is the library's to check)
    call = _bound(_without_trace("parrot_cache8_plan"),
                  (ctypes.byref(p), ctypes.byref(rows), query_offsets, prefix_lens, prefix_parents, suffix_lens, group_ids,
                   plan, 0 if plan is None else plan.numel() * 4), _device(query_offsets), stream)
    return call


class _without_trace:
    """A C entry point that takes a stream but no trace, called as one that takes both."""

    def __init__(self, name: str):
        self.fn = getattr(load_library(), name)
        self.argtypes = self.fn.argtypes

    def __call__(self, *args):
        return self.fn(*args[:-1])


def parrot_cache8_plan(problem, rows, query_offsets, prefix_lens, prefix_parents, suffix_lens, group_ids, plan,
                       stream=None):
    """The plan of a step (see the C header); prefix_parents None: flat groups."""
    _plan_call(problem, rows, query_offsets, prefix_lens, prefix_parents, suffix_lens, group_ids, plan, stream)()


def _attend_call(problem, rows, q, query_offsets, prefix, suffix, prefix_tables, prefix_lens, prefix_parents, suffix_tables,
                 suffix_lens, group_ids, plan, out, lse, workspace, stream):
    p, T, HQ, dt = problem, rows.num_query_rows, rows.num_query_heads, _TORCH_DTYPES[problem.dtype]
    for x, name, dtype, least in ((q, "q", dt, T * HQ * p.head_dim), (out, "out", dt, T * HQ * p.head_dim),
                                  (lse, "lse", torch.float32, T * HQ), (plan, "plan", torch.int32, 0)):
        _need(x, name, dtype, least, q.device)
    _need_tree(p, q.device, query_offsets, None, prefix_tables, prefix_lens, prefix_parents, suffix_tables, suffix_lens,
               group_ids)
    if isinstance(workspace, torch.Tensor):          # (its size is the library's to check)
        _need(workspace, "workspace", workspace.dtype, 0, q.device)
    own = _pool(suffix, "suffix", p.num_suffix_blocks, p, q.device)
    pre = _pool(prefix, "prefix", p.num_prefix_blocks, p, q.device) if p.num_groups > 0 else None
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    call = _bound(load_library().parrot_cache8_attention,
                  (ctypes.byref(p), ctypes.byref(rows), q, query_offsets, None if pre is None else ctypes.byref(pre),
                   ctypes.byref(own), prefix_tables, prefix_lens, prefix_parents, suffix_tables, suffix_lens, group_ids, plan,
                   0 if plan is None else plan.numel() * 4, out, lse, workspace, ws_bytes), _device(q), stream)
    call.pools = (prefix, suffix)                # (the structs hold addresses only)
    return call


def parrot_cache8_attention(problem, rows, q, query_offsets, prefix, suffix, prefix_block_tables, prefix_lens, prefix_parents,
                            suffix_block_tables, suffix_lens, group_ids, plan, out, lse, workspace, stream=None, trace=None):
    """Attention of a step's rows over a layer's 8-bit pools (see the C header);
    prefix_parents None: flat groups."""
    _attend_call(problem, rows, q, query_offsets, prefix, suffix, prefix_block_tables, prefix_lens, prefix_parents,
                 suffix_block_tables, suffix_lens, group_ids, plan, out, lse, workspace, stream)(trace)


def parrot_validate_cache8_inputs(problem, rows, query_offsets, prefix_block_tables, prefix_lens, prefix_parents,
                                  suffix_block_tables, suffix_lens, group_ids, scratch, stream=None):
    """Device-side content check of a step's inputs (synchronises)."""
    _need_tree(problem, suffix_lens.device, query_offsets, None, prefix_block_tables, prefix_lens, prefix_parents,
               suffix_block_tables, suffix_lens, group_ids)
    _need(scratch, "scratch", torch.int32, 16, suffix_lens.device)
    with torch.cuda.device(_device(suffix_lens)):
        _check(load_library().parrot_validate_cache8_inputs(
            ctypes.byref(problem), ctypes.byref(rows), _ptr(query_offsets), _ptr(prefix_block_tables), _ptr(prefix_lens),
            _ptr(prefix_parents), _ptr(suffix_block_tables), _ptr(suffix_lens), _ptr(group_ids), _ptr(scratch),
            _stream(stream, suffix_lens.device)))


def _copy_call(pools, num_blocks, src, dst, num_copies, stream):
    device = _device(src)
    n = int(num_copies)
    for x, name in ((src, "src"), (dst, "dst")):
        _need(x, name, torch.int32, n, device)
    array = (ParrotBlockPool * max(len(pools), 1))()
    for i, t in enumerate(pools):
        if not t.is_contiguous() or t.dim() < 1 or t.shape[0] < num_blocks:
            raise ValueError(f"pool {i} is not a contiguous tensor of at least {num_blocks} blocks")
        if t.device != device:
            raise ValueError(f"pool {i} is on {t.device}, not on {device}")
        array[i] = ParrotBlockPool(t.data_ptr(), t[0].numel() * t.element_size())
    if len({t.data_ptr() for t in pools}) < len(pools):
        raise ValueError("a pool is listed twice")
    call = _bound(load_library().parrot_copy_blocks, (array, len(pools), int(num_blocks), src, dst, n), device, stream)
    call.pools = list(pools)                     # (the structs hold addresses only)
    return call


def parrot_copy_blocks(pools, num_blocks, src, dst, num_copies, stream=None, trace=None):
    """Block dst[i] of every pool becomes block src[i] (see the C header); pools: tensors
    whose first dimension counts blocks."""
    _copy_call(pools, num_blocks, src, dst, num_copies, stream)(trace)


# -------------------------------------------------------------------- handles
class Cache8Filler:
    """Owns the rotated queries of one fill shape: up to ``num_query_rows`` rows, at
    most ``max_query_rows`` per request.  ``num_query_heads`` 0: keys and values only."""

    def __init__(self, problem: ParrotProblem, num_query_rows: int, max_query_rows: int, num_query_heads: int, *,
                 rotary: Optional[ParrotRotary] = None, norm_eps: float = 0.0, device="cuda"):
        self.problem = problem
        self.counts = (int(num_query_rows), int(max_query_rows), int(num_query_heads))
        self.rotary = rotary
        self.norm_eps = float(norm_eps)
        T, _, HQ = self.counts
        self.q_out = None if HQ == 0 else torch.empty((T, HQ, problem.head_dim), device=device,
                                                      dtype=_TORCH_DTYPES[problem.dtype])

    def bind(self, t: dict, stream=None):
        """Marshal once; the returned callable re-issues the same call.  ``t`` holds
        q_rows, k_rows, v_rows, positions, query_offsets, suffix_tables, suffix_lens, the
        layer's pools ``suffix`` and optionally q_norm, k_norm."""
        return _fill_call(self.problem, *self.counts, self.rotary, self.norm_eps,
                          t["q_rows"] if self.q_out is not None else None, t["k_rows"], t["v_rows"], t.get("q_norm"),
                          t.get("k_norm"), t.get("positions"), t["query_offsets"], t["suffix_tables"],
                          t["suffix_lens"], self.q_out, t["suffix"], stream)

    def __call__(self, t: dict, stream=None, trace=None):
        self.bind(t, stream=stream)(trace)
        return self.q_out


class Cache8Planner:
    """Owns the plan of one batch shape, which every layer's ``Cache8Decoder`` reads."""

    def __init__(self, problem: ParrotProblem, rows: ParrotTreeRows, nested: bool = False, device="cuda"):
        self.problem, self.rows, self.nested = problem, rows, bool(nested)
        self.device = torch.device(device)
        with torch.cuda.device(self.device):     # the sizes depend on the device
            self.plan_bytes = parrot_cache8_plan_bytes(problem, rows)
            self.workspace_bytes = parrot_cache8_workspace_bytes(problem, rows)
        self.plan = torch.empty(max(self.plan_bytes, 256) // 4, dtype=torch.int32, device=device)

    def bind(self, t: dict, stream=None):
        """Marshal once; the returned callable writes the plan of what ``t``'s int arrays hold
        then: query_offsets, suffix_lens, group_ids, prefix_lens, and prefix_parents where the
        planner is ``nested``."""
        return _plan_call(self.problem, self.rows, t["query_offsets"], t.get("prefix_lens"),
                          t["prefix_parents"] if self.nested else None, t["suffix_lens"], t["group_ids"], self.plan, stream)

    def __call__(self, t: dict, stream=None):
        self.bind(t, stream=stream)()
        return self.plan


class Cache8Decoder:
    """Owns the output and lse of one layer, and a workspace unless it is given one (layers
    that run one after another may share it)."""

    def __init__(self, planner: Cache8Planner, workspace: Optional[torch.Tensor] = None):
        self.planner = planner
        p, T, HQ = planner.problem, planner.rows.num_query_rows, planner.rows.num_query_heads
        self.out = torch.empty((T, HQ, p.head_dim), dtype=_TORCH_DTYPES[p.dtype], device=planner.device)
        self.lse = torch.empty((T, HQ), dtype=torch.float32, device=planner.device)
        self.workspace = workspace if workspace is not None else \
            torch.empty(max(planner.workspace_bytes, 256), dtype=torch.uint8, device=planner.device)

    def bind(self, t: dict, stream=None):
        """Marshal once; the returned callable re-issues the same call, with what the plan
        holds then.  ``t`` holds the planner's int arrays, q_rows, suffix_tables, the layer's
        pools ``suffix`` and, with groups, prefix_tables and ``prefix``."""
        pl = self.planner
        return _attend_call(pl.problem, pl.rows, t["q_rows"], t["query_offsets"], t.get("prefix"), t["suffix"],
                            t.get("prefix_tables"), t.get("prefix_lens"), t["prefix_parents"] if pl.nested else None,
                            t["suffix_tables"], t["suffix_lens"], t["group_ids"], pl.plan, self.out, self.lse,
                            self.workspace, stream)

    def __call__(self, t: dict, stream=None, trace=None):
        self.bind(t, stream=stream)(trace)
        return self.out, self.lse


class BlockCopier:
    """Copies blocks of the pools of all layers (tensors whose first dimension counts blocks),
    up to ``num_copies`` at once."""

    def __init__(self, pools, num_copies: int):
        self.pools = list(pools)
        self.num_copies = int(num_copies)
        self.num_blocks = min((t.shape[0] for t in self.pools), default=1)

    def bind(self, src: torch.Tensor, dst: torch.Tensor, stream=None):
        """Marshal once; the returned callable re-issues the same call.  ``src`` and ``dst`` are
        int32 tensors of ``num_copies`` block ids (-1: no copy)."""
        return _copy_call(self.pools, self.num_blocks, src, dst, self.num_copies, stream)

    def __call__(self, src: torch.Tensor, dst: torch.Tensor, stream=None, trace=None):
        self.bind(src, dst, stream=stream)(trace)


# ------------------------------------------------------------- one-call forms
# With ``stream``, the host copies of lengths, the results' memory and the call itself are that
# stream's: inputs may come from work that it holds, and a result may be dropped at once.
def cache8_fill(q_rows, k_rows, v_rows, positions, query_offsets, suffix, suffix_tables, suffix_lens, *, rotary=None,
                q_norm=None, k_norm=None, norm_eps=0.0, stream=None):
    """One fill on torch tensors: returns the rotated queries [T, HQ, D] (None without
    q_rows) and writes keys and values into the pools.  Sizes the call from host copies
    of the offsets and lengths; engines that know them reuse a Cache8Filler."""
    with _on_stream(stream, k_rows.device):
        blocks, heads, block, dim = suffix["k"].shape
        prob = make_problem(num_requests=suffix_lens.shape[0], num_heads=heads, head_dim=dim, block_size=block,
                            num_groups=0, max_group_size=0, max_prefix_len=0,
                            max_suffix_len=max(1, int(suffix_lens.max()) if suffix_lens.numel() else 0),
                            prefix_table_stride=0, suffix_table_stride=suffix_tables.shape[1], num_prefix_blocks=0,
                            num_suffix_blocks=blocks, dtype=k_rows.dtype, sm_scale=1.0)
        fill = Cache8Filler(prob, k_rows.shape[0], _most_rows(query_offsets), 0 if q_rows is None else q_rows.shape[1],
                            rotary=rotary, norm_eps=norm_eps, device=k_rows.device)
        return fill(dict(q_rows=q_rows, k_rows=k_rows, v_rows=v_rows, positions=positions, query_offsets=query_offsets,
                         suffix=suffix, suffix_tables=suffix_tables, suffix_lens=suffix_lens, q_norm=q_norm,
                         k_norm=k_norm), stream=stream)


def cache8_attention(q_rows, query_offsets, prefix, suffix, prefix_tables, prefix_lens, suffix_tables, suffix_lens,
                     group_ids, *, sm_scale=None, prefix_parents=None, stream=None):
    """One plan and one layer's attention on torch tensors; q_rows [T, HQ, D] with HQ a multiple
    of the pools' heads.  Without groups ``prefix``, ``prefix_tables`` and ``prefix_lens`` may be
    None.  Returns (out, lse)."""
    sm_scale = 1.0 / math.sqrt(q_rows.shape[-1]) if sm_scale is None else sm_scale
    with _on_stream(stream, q_rows.device):
        k = suffix["k"]
        like = k.view(torch.uint8).new_empty((), dtype=q_rows.dtype).expand(k.shape)       # (shape and type only)
        none = prefix is None
        empty = lambda *shape: torch.empty(shape, dtype=torch.int32, device=q_rows.device)
        prefix_lens = empty(0) if prefix_lens is None else prefix_lens
        prefix_tables = empty(0, 0) if prefix_tables is None else prefix_tables
        pre = like if none else like[:1].expand(prefix["k"].shape[0], *k.shape[1:])
        prob = _sizes_from_tensors(like.transpose(1, 2), pre, like, prefix_tables, suffix_tables, group_ids, prefix_lens,
                                   suffix_lens, sm_scale, prefix_parents)
        rows = tree_rows_from_host(query_offsets.cpu().numpy(), group_ids.cpu().numpy(), prob.num_groups, q_rows.shape[1],
                                   None if prefix_parents is None else prefix_parents.cpu().numpy())
        rows.num_query_rows = q_rows.shape[0]
        rows.max_query_rows = max(1, rows.max_query_rows)
        plan = Cache8Planner(prob, rows, nested=prefix_parents is not None, device=q_rows.device)
        dec = Cache8Decoder(plan)
        t = dict(q_rows=q_rows, query_offsets=query_offsets, prefix=prefix, suffix=suffix, prefix_tables=prefix_tables,
                 prefix_lens=prefix_lens, suffix_tables=suffix_tables, suffix_lens=suffix_lens, group_ids=group_ids,
                 prefix_parents=prefix_parents)
        plan(t, stream=stream)
        return dec(t, stream=stream)


def copy_blocks(pools, src, dst, *, stream=None):
    """Block dst[i] of every pool (tensors whose first dimension counts blocks) becomes block
    src[i].  ``src`` and ``dst`` are int32 tensors on the GPU (-1: no copy), or sequences on the
    host, whose ids and overlaps are then checked."""
    pools = list(pools)
    if not pools:
        return
    device = _device(pools[0])
    with _on_stream(stream, device):
        if not isinstance(src, torch.Tensor):
            a, b = [int(x) for x in src], [int(x) for x in dst]
            most = min(t.shape[0] for t in pools)
            if len(a) != len(b):
                raise ValueError(f"{len(a)} source and {len(b)} destination blocks")
            if any(not 0 <= x < most for x in a + b):
                raise ValueError(f"a block id is not in [0, {most})")
            if len(set(b)) < len(b) or set(a) & set(b):
                raise ValueError("a destination is also another copy's source or destination")
            src, dst = (torch.tensor(x, dtype=torch.int32, device=device) for x in (a, b))
        if src.shape != dst.shape:
            raise ValueError("src and dst differ in shape")
        BlockCopier(pools, src.numel())(src, dst, stream=stream)
