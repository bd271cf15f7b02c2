"""A drafting step through libparrot_attn (argument marshalling only): fill of new
rows (norm, rotation, cache write), attention for trees of drafted tokens, the
accepted tokens and their move in the cache.

The ``parrot_*`` functions forward to the C entry points of the same name in
``include/parrot_attn.h``; ``RotaryFiller``, ``TreeDecoder`` and ``TreeVerifier`` keep the
output buffers of one batch shape and bind a call once; ``rotary_fill``,
``tree_decode``, ``tree_accept`` and ``tree_commit`` are one-call forms on torch tensors.

A step of an engine that verifies drafted trees, per layer: ``RotaryFiller`` with the
drafted rows' projections, then ``TreeDecoder``; after the last layer, with the model's
choice at every row, ``TreeVerifier.bind_accept`` once and ``bind_commit`` per layer.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from .binding import (DTYPE_CODES, PARROT_ERR_INVALID_ARGUMENT, ParrotError, ParrotFillRows, ParrotProblem,
                      ParrotRotary, ParrotRotaryConfig, ParrotTrace, ParrotTreeRows, _check, _on_stream, _ptr,
                      _sizes_from_tensors, load_library, make_problem, parrot_last_error)

_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "wavelength": 4}


def make_rotary(rotary_dim: int, *, base: float = 10000.0, interleaved: bool = False, scaling: str = "none",
                factor: float = 1.0, original_length: float = 0.0, low: float = 0.0, high: float = 0.0,
                amplitude: float = 0.0) -> ParrotRotary:
    """The rotary embedding of a model (see parrot_rotary_config in the C header);
    ``scaling`` is none, linear, ntk, yarn or wavelength."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling {scaling!r} is not one of {sorted(_SCALINGS)}")
    out = ParrotRotary()
    cfg = ParrotRotaryConfig(int(rotary_dim), int(bool(interleaved)), float(base), _SCALINGS[scaling], float(factor),
                             float(original_length), float(low), float(high), float(amplitude))
    _check(load_library().parrot_rotary_init(ctypes.byref(out), ctypes.byref(cfg)))
    return out


def rotary_from_frequencies(radians, *, interleaved: bool = False, amplitude: float = 1.0) -> ParrotRotary:
    """A rotary embedding from the angle per position of every pair (a sequence)."""
    f = (ctypes.c_double * len(radians))(*[float(x) for x in radians])
    out = ParrotRotary()
    _check(load_library().parrot_rotary_from_frequencies(ctypes.byref(out), 2 * len(f), int(bool(interleaved)), f,
                                                         float(amplitude)))
    return out


def make_tree_rows(num_query_rows, max_query_rows, max_group_rows, num_query_heads) -> ParrotTreeRows:
    return ParrotTreeRows(int(num_query_rows), int(max_query_rows), int(max_group_rows), int(num_query_heads))


def tree_rows_from_host(query_offsets, group_ids, num_groups, num_query_heads, prefix_parents=None) -> ParrotTreeRows:
    """Row counts of a tree call from host copies of its offsets and groups."""
    from .binding import prefill_rows_from_host
    r = prefill_rows_from_host(query_offsets, group_ids, num_groups, prefix_parents)
    return make_tree_rows(r.num_query_rows, r.max_query_rows, r.max_group_rows, num_query_heads)


def parrot_tree_workspace_bytes(problem: ParrotProblem, rows: ParrotTreeRows) -> int:
    n = load_library().parrot_tree_workspace_bytes(ctypes.byref(problem), ctypes.byref(rows))
    if n == ctypes.c_size_t(-1).value:
        raise ParrotError(PARROT_ERR_INVALID_ARGUMENT, parrot_last_error())
    return int(n)


# ---------------------------------------------------------------- marshalling
_TORCH_DTYPES = {v: k for k, v in DTYPE_CODES.items()}


def _stream(stream, device: torch.device) -> int:
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _device(t: torch.Tensor) -> torch.device:
    if t.device.type != "cuda":
        raise ValueError("the library takes tensors on the GPU")
    return t.device


def _bound(fn, values, device: torch.device, stream):
    """A callable that issues ``fn(*values, stream, trace)`` with ``device`` current; the
    arguments are converted to their C types once, and the tensors kept alive."""
    args = [t(_ptr(v)) if isinstance(v, (int, torch.Tensor)) else v
            for t, v in zip(fn.argtypes, (*values, _stream(stream, device)))]
    index = device.index if device.index is not None else torch.cuda.current_device()

    def call(trace: Optional[ParrotTrace] = None):
        t = ctypes.byref(trace) if trace is not None else None
        if torch.cuda.current_device() == index:
            status = fn(*args, t)
        else:
            with torch.cuda.device(index):
                status = fn(*args, t)
        if status:
            _check(status)
    call.holds = values
    return call


def _need(t, name: str, dtype: torch.dtype, least: int, device: torch.device):
    """Refuses a tensor that the kernels would read or write beyond its end (addresses
    and None go to the library's own checks)."""
    if not isinstance(t, torch.Tensor):
        return
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < least:
        raise ValueError(f"{name} is not a contiguous {dtype} tensor of at least {least} elements")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")


def _need_cache(p: ParrotProblem, device: torch.device, suffix_k, suffix_v, suffix_tables, suffix_lens):
    own = p.num_suffix_blocks * p.num_heads * p.block_size * p.head_dim
    for t, name in ((suffix_k, "suffix_k"), (suffix_v, "suffix_v")):
        _need(t, name, _TORCH_DTYPES[p.dtype], own, device)
    _need(suffix_tables, "suffix_tables", torch.int32, p.num_requests * p.suffix_table_stride, device)
    _need(suffix_lens, "suffix_lens", torch.int32, p.num_requests, device)


def _need_tree(p: ParrotProblem, device: torch.device, query_offsets, tree_parents, prefix_tables, prefix_lens,
               prefix_parents, suffix_tables, suffix_lens, group_ids):
    """The int arrays of a tree call."""
    arrays = [(query_offsets, "query_offsets", p.num_requests + 1), (tree_parents, "tree_parents", 0),
              (group_ids, "group_ids", p.num_requests), (suffix_lens, "suffix_lens", p.num_requests),
              (suffix_tables, "suffix_tables", p.num_requests * p.suffix_table_stride)]
    if p.num_groups > 0:
        arrays += [(prefix_lens, "prefix_lens", p.num_groups), (prefix_parents, "prefix_parents", p.num_groups),
                   (prefix_tables, "prefix_tables", p.num_groups * p.prefix_table_stride)]
    for x, name, least in arrays:
        _need(x, name, torch.int32, least, device)


def _need_rows(x, name: str, rows: int, heads: int, p: ParrotProblem, device: torch.device):
    """Rows [rows, heads, D] of any row stride."""
    if not isinstance(x, torch.Tensor):
        return
    if x.dtype != _TORCH_DTYPES[p.dtype] or x.dim() != 3 or x.shape[0] < rows or tuple(x.shape[1:]) != (heads, p.head_dim):
        raise ValueError(f"{name} is not [{rows}, {heads}, {p.head_dim}] of {_TORCH_DTYPES[p.dtype]}")
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, not on {device}")


def _within_parents(rows: ParrotTreeRows, tree_parents) -> ParrotTreeRows:
    """The row counts of a call whose parents may stop where its padding begins: only the
    device knows where that is, so rows behind the tensor's end are taken as padding, and
    nothing is read there whatever the offsets say."""
    if not isinstance(tree_parents, torch.Tensor) or tree_parents.numel() >= rows.num_query_rows:
        return rows
    n = tree_parents.numel()
    return make_tree_rows(n, rows.max_query_rows, min(rows.max_group_rows, n), rows.num_query_heads)


def _row_stride(x: torch.Tensor, name: str) -> int:
    """Elements between the rows of [rows, heads, D] whose heads are adjacent."""
    if x.dim() != 3 or x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != x.shape[2]):
        raise ValueError(f"{name} is not [rows, heads, head_dim] with adjacent heads")
    return x.stride(0) if x.shape[0] > 1 else x.shape[1] * x.shape[2]


def _fill_call(problem, num_query_rows, max_query_rows, num_query_heads, rotary, norm_eps, q, k, v, q_norm, k_norm,
               positions, query_offsets, suffix_tables, suffix_lens, q_out, suffix_k, suffix_v, stream):
    fn = load_library().parrot_rotary_fill
    T, D, dt = int(num_query_rows), problem.head_dim, _TORCH_DTYPES[problem.dtype]
    for x, name, heads in ((q, "q", int(num_query_heads)), (k, "k", problem.num_heads), (v, "v", problem.num_heads)):
        _need_rows(x, name, T, heads, problem, k.device)
    _need(q_out, "q_out", dt, T * int(num_query_heads) * D, k.device)
    for x, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        _need(x, name, dt, D, k.device)
    _need(positions, "positions", torch.int32, T, k.device)
    _need(query_offsets, "query_offsets", torch.int32, problem.num_requests + 1, k.device)
    _need_cache(problem, k.device, suffix_k, suffix_v, suffix_tables, suffix_lens)
    rows = ParrotFillRows(int(num_query_rows), int(max_query_rows), int(num_query_heads), float(norm_eps),
                          0 if q is None else _row_stride(q, "q"), _row_stride(k, "k"), _row_stride(v, "v"))
    return _bound(fn, (ctypes.byref(problem), ctypes.byref(rows), None if rotary is None else ctypes.byref(rotary), q,
                       k, v, q_norm, k_norm, positions, query_offsets, suffix_tables, suffix_lens, q_out, suffix_k,
                       suffix_v), _device(k), stream)


def parrot_rotary_fill(problem, num_query_rows, max_query_rows, num_query_heads, rotary, q, k, v, q_norm, k_norm,
                       positions, query_offsets, suffix_tables, suffix_lens, q_out, suffix_k, suffix_v,
                       norm_eps=0.0, stream=None, trace=None):
    """Norm, rotate and cache new rows (see the C header).  The row strides come from
    q, k and v ([rows, heads, D], heads adjacent); q and q_out may be None."""
    _fill_call(problem, num_query_rows, max_query_rows, num_query_heads, rotary, norm_eps, q, k, v, q_norm, k_norm,
               positions, query_offsets, suffix_tables, suffix_lens, q_out, suffix_k, suffix_v, stream)(trace)


def _tree_call(problem, rows, q, query_offsets, tree_parents, prefix_k, prefix_v, suffix_k, suffix_v, prefix_tables,
               prefix_lens, prefix_parents, suffix_tables, suffix_lens, group_ids, out, lse, workspace, stream):
    fn = load_library().parrot_shared_prefix_tree_decode
    p, T, HQ, dt = problem, rows.num_query_rows, rows.num_query_heads, _TORCH_DTYPES[problem.dtype]
    for x, name, dtype, least in ((q, "q", dt, T * HQ * p.head_dim), (out, "out", dt, T * HQ * p.head_dim),
                                  (lse, "lse", torch.float32, T * HQ)):
        _need(x, name, dtype, least, q.device)
    _need_tree(p, q.device, query_offsets, tree_parents, prefix_tables, prefix_lens, prefix_parents, suffix_tables,
               suffix_lens, group_ids)
    if p.num_groups > 0:
        for x, name in ((prefix_k, "prefix_k"), (prefix_v, "prefix_v")):
            _need(x, name, dt, p.num_prefix_blocks * p.num_heads * p.block_size * p.head_dim, q.device)
    if isinstance(workspace, torch.Tensor):          # (its size is the library's to check)
        _need(workspace, "workspace", workspace.dtype, 0, q.device)
    rows = _within_parents(rows, tree_parents)
    _need_cache(p, q.device, suffix_k, suffix_v, suffix_tables, suffix_lens)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return _bound(fn, (ctypes.byref(problem), ctypes.byref(rows), q, query_offsets, tree_parents, prefix_k, prefix_v,
                       suffix_k, suffix_v, prefix_tables, prefix_lens, prefix_parents, suffix_tables, suffix_lens,
                       group_ids, out, lse, workspace, ws_bytes), _device(q), stream)


def parrot_shared_prefix_tree_decode(problem, rows, q, query_offsets, tree_parents, prefix_k, prefix_v, suffix_k,
                                     suffix_v, prefix_block_tables, prefix_lens, prefix_parents, suffix_block_tables,
                                     suffix_lens, group_ids, out, lse, workspace, stream=None, trace=None):
    """Attention of drafted trees (see the C header); tree_parents None: chains,
    prefix_parents None: flat groups.  Rows behind the end of tree_parents are padding."""
    _tree_call(problem, rows, q, query_offsets, tree_parents, prefix_k, prefix_v, suffix_k, suffix_v,
               prefix_block_tables, prefix_lens, prefix_parents, suffix_block_tables, suffix_lens, group_ids, out,
               lse, workspace, stream)(trace)


def parrot_validate_tree_inputs(problem, rows, query_offsets, tree_parents, prefix_block_tables, prefix_lens,
                                prefix_parents, suffix_block_tables, suffix_lens, group_ids, scratch, stream=None):
    """Device-side content check of a tree call's inputs (synchronises)."""
    _need_tree(problem, suffix_lens.device, query_offsets, tree_parents, prefix_block_tables, prefix_lens,
               prefix_parents, suffix_block_tables, suffix_lens, group_ids)
    _need(scratch, "scratch", torch.int32, 16, suffix_lens.device)
    rows = _within_parents(rows, tree_parents)
    with torch.cuda.device(_device(suffix_lens)):
        _check(load_library().parrot_validate_tree_inputs(
            ctypes.byref(problem), ctypes.byref(rows), _ptr(query_offsets), _ptr(tree_parents),
            _ptr(prefix_block_tables), _ptr(prefix_lens), _ptr(prefix_parents), _ptr(suffix_block_tables),
            _ptr(suffix_lens), _ptr(group_ids), _ptr(scratch), _stream(stream, suffix_lens.device)))


def _accept_call(num_requests, rows, query_offsets, tree_parents, draft_tokens, target_tokens, root_tokens,
                 accept_rows, accept_lens, next_tokens, stream):
    fn = load_library().parrot_tree_accept
    T, R = rows.num_query_rows, int(num_requests)
    for x, name, least in ((query_offsets, "query_offsets", R + 1), (tree_parents, "tree_parents", 0),
                           (draft_tokens, "draft_tokens", T), (target_tokens, "target_tokens", T),
                           (root_tokens, "root_tokens", R), (accept_rows, "accept_rows", T),
                           (accept_lens, "accept_lens", R), (next_tokens, "next_tokens", R)):
        _need(x, name, torch.int32, least, query_offsets.device)
    rows = _within_parents(rows, tree_parents)
    return _bound(fn, (int(num_requests), ctypes.byref(rows), query_offsets, tree_parents, draft_tokens,
                       target_tokens, root_tokens, accept_rows, accept_lens, next_tokens), _device(query_offsets),
                  stream)


def parrot_tree_accept(num_requests, rows, query_offsets, tree_parents, draft_tokens, target_tokens, root_tokens,
                       accept_rows, accept_lens, next_tokens, stream=None, trace=None):
    """The drafted tokens a greedy model agrees with (see the C header)."""
    _accept_call(num_requests, rows, query_offsets, tree_parents, draft_tokens, target_tokens, root_tokens,
                 accept_rows, accept_lens, next_tokens, stream)(trace)


def _commit_call(problem, rows, query_offsets, accept_rows, accept_lens, suffix_tables, suffix_lens, suffix_k,
                 suffix_v, committed_lens, stream):
    fn = load_library().parrot_tree_commit
    R = problem.num_requests
    for x, name, least in ((query_offsets, "query_offsets", R + 1), (accept_rows, "accept_rows", rows.num_query_rows),
                           (accept_lens, "accept_lens", R), (committed_lens, "committed_lens", R)):
        _need(x, name, torch.int32, least, suffix_k.device)
    _need_cache(problem, suffix_k.device, suffix_k, suffix_v, suffix_tables, suffix_lens)
    return _bound(fn, (ctypes.byref(problem), ctypes.byref(rows), query_offsets, accept_rows, accept_lens,
                       suffix_tables, suffix_lens, suffix_k, suffix_v, committed_lens), _device(suffix_k), stream)


def parrot_tree_commit(problem, rows, query_offsets, accept_rows, accept_lens, suffix_tables, suffix_lens, suffix_k,
                       suffix_v, committed_lens, stream=None, trace=None):
    """Move the accepted tokens' keys and values into cache order (see the C header)."""
    _commit_call(problem, rows, query_offsets, accept_rows, accept_lens, suffix_tables, suffix_lens, suffix_k,
                 suffix_v, committed_lens, stream)(trace)


# -------------------------------------------------------------------- handles
class RotaryFiller:
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
        pools (suffix_k / suffix_v or k_pool / v_pool) and optionally q_norm, k_norm."""
        return _fill_call(self.problem, *self.counts, self.rotary, self.norm_eps,
                          t["q_rows"] if self.q_out is not None else None, t["k_rows"], t["v_rows"], t.get("q_norm"),
                          t.get("k_norm"), t.get("positions"), t["query_offsets"], t["suffix_tables"],
                          t["suffix_lens"], self.q_out, t.get("suffix_k", t.get("k_pool")),
                          t.get("suffix_v", t.get("v_pool")), stream)

    def __call__(self, t: dict, stream=None, trace=None):
        self.bind(t, stream=stream)(trace)
        return self.q_out


class TreeDecoder:
    """Owns the output, lse and workspace buffers of one tree-decode shape."""

    def __init__(self, problem: ParrotProblem, rows: ParrotTreeRows, device="cuda"):
        self.problem = problem
        self.rows = rows
        T, HQ = rows.num_query_rows, rows.num_query_heads
        with torch.cuda.device(device):          # the workspace depends on the device
            nbytes = parrot_tree_workspace_bytes(problem, rows)
        self.out = torch.empty((T, HQ, problem.head_dim), dtype=_TORCH_DTYPES[problem.dtype], device=device)
        self.lse = torch.empty((T, HQ), dtype=torch.float32, device=device)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)

    def bind(self, t: dict, stream=None, nested: bool = False):
        """Marshal once; the returned callable re-issues the same call.  ``t`` holds
        q_rows, query_offsets, tree_parents (absent or None: chains), the pools and
        the int arrays as for Prefiller; ``nested`` passes t["prefix_parents"]."""
        k, v = t.get("k_pool"), t.get("v_pool")
        return _tree_call(self.problem, self.rows, t["q_rows"], t["query_offsets"], t.get("tree_parents"),
                          t.get("prefix_k", k), t.get("prefix_v", v), t.get("suffix_k", k), t.get("suffix_v", v),
                          t.get("prefix_tables"), t.get("prefix_lens"), t["prefix_parents"] if nested else None,
                          t["suffix_tables"], t["suffix_lens"], t["group_ids"], self.out, self.lse, self.workspace,
                          stream)

    def __call__(self, t: dict, stream=None, trace=None, nested: bool = False):
        self.bind(t, stream=stream, nested=nested)(trace)
        return self.out, self.lse


class TreeVerifier:
    """Owns the accepted rows, their counts, the next tokens and the committed lengths
    of one batch shape."""

    def __init__(self, problem: ParrotProblem, rows: ParrotTreeRows, device="cuda"):
        self.problem = problem
        self.rows = rows
        ints = lambda n: torch.empty(n, dtype=torch.int32, device=device)
        self.accept_rows = ints(rows.num_query_rows)
        self.accept_lens, self.next_tokens, self.committed_lens = (ints(problem.num_requests) for _ in range(3))

    def bind_accept(self, t: dict, stream=None):
        """The walk over t's tree_parents (absent or None: chains), draft_tokens,
        target_tokens and root_tokens; fills accept_rows, accept_lens, next_tokens."""
        return _accept_call(self.problem.num_requests, self.rows, t["query_offsets"], t.get("tree_parents"),
                            t["draft_tokens"], t["target_tokens"], t["root_tokens"], self.accept_rows,
                            self.accept_lens, self.next_tokens, stream)

    def bind_commit(self, t: dict, stream=None):
        """The move of one layer's accepted rows: t's accept_rows and accept_lens, or this
        verifier's own; fills committed_lens."""
        return _commit_call(self.problem, self.rows, t["query_offsets"], t.get("accept_rows", self.accept_rows),
                            t.get("accept_lens", self.accept_lens), t["suffix_tables"], t["suffix_lens"],
                            t.get("suffix_k", t.get("k_pool")), t.get("suffix_v", t.get("v_pool")),
                            self.committed_lens, stream)


# ------------------------------------------------------------- one-call forms
# With ``stream``, the host copies of lengths, the results' memory and the call itself are that
# stream's: inputs may come from work that it holds, and a result may be dropped at once.
def _cache_problem(suffix_k, suffix_tables, suffix_lens) -> ParrotProblem:
    """ParrotProblem of a call that touches own tokens only (one device-to-host copy
    of the lengths, for their maximum)."""
    blocks, heads, block, dim = suffix_k.shape
    return make_problem(num_requests=suffix_lens.shape[0], num_heads=heads, head_dim=dim, block_size=block,
                        num_groups=0, max_group_size=0, max_prefix_len=0,
                        max_suffix_len=max(1, int(suffix_lens.max()) if suffix_lens.numel() else 0),
                        prefix_table_stride=0, suffix_table_stride=suffix_tables.shape[1], num_prefix_blocks=0,
                        num_suffix_blocks=blocks, dtype=suffix_k.dtype, sm_scale=1.0)


def _most_rows(query_offsets) -> int:
    off = query_offsets.cpu()
    return max(1, int((off[1:] - off[:-1]).max())) if off.numel() > 1 else 1


def rotary_fill(q_rows, k_rows, v_rows, positions, query_offsets, suffix_k, suffix_v, suffix_tables, suffix_lens, *,
                rotary=None, q_norm=None, k_norm=None, norm_eps=0.0, stream=None):
    """One fill on torch tensors: returns the rotated queries [T, HQ, D] (None without
    q_rows) and writes keys and values into the pools.  Sizes the call from host copies
    of the offsets and lengths; engines that know them reuse a RotaryFiller."""
    with _on_stream(stream, k_rows.device):
        prob = _cache_problem(suffix_k, suffix_tables, suffix_lens)
        fill = RotaryFiller(prob, k_rows.shape[0], _most_rows(query_offsets), 0 if q_rows is None else q_rows.shape[1],
                            rotary=rotary, norm_eps=norm_eps, device=k_rows.device)
        return fill(dict(q_rows=q_rows, k_rows=k_rows, v_rows=v_rows, positions=positions, query_offsets=query_offsets,
                         suffix_k=suffix_k, suffix_v=suffix_v, suffix_tables=suffix_tables, suffix_lens=suffix_lens,
                         q_norm=q_norm, k_norm=k_norm), stream=stream)


def tree_decode(q_rows, query_offsets, tree_parents, prefix_k, prefix_v, suffix_k, suffix_v, prefix_tables,
                prefix_lens, suffix_tables, suffix_lens, group_ids, *, sm_scale=None, prefix_parents=None, stream=None):
    """One tree-decode call on torch tensors (see TreeDecoder); q_rows [T, HQ, D] with HQ
    a multiple of the pools' heads.  Returns (out, lse)."""
    sm_scale = 1.0 / math.sqrt(q_rows.shape[-1]) if sm_scale is None else sm_scale
    with _on_stream(stream, q_rows.device):
        prob = _sizes_from_tensors(suffix_k.transpose(1, 2), prefix_k, suffix_k, prefix_tables, suffix_tables, group_ids,
                                   prefix_lens, suffix_lens, sm_scale, prefix_parents)
        rows = tree_rows_from_host(query_offsets.cpu().numpy(), group_ids.cpu().numpy(), prob.num_groups, q_rows.shape[1],
                                   None if prefix_parents is None else prefix_parents.cpu().numpy())
        rows.num_query_rows = q_rows.shape[0]
        dec = TreeDecoder(prob, rows, device=q_rows.device)
        return dec(dict(q_rows=q_rows, query_offsets=query_offsets, tree_parents=tree_parents, prefix_k=prefix_k,
                        prefix_v=prefix_v, suffix_k=suffix_k, suffix_v=suffix_v, prefix_tables=prefix_tables,
                        prefix_lens=prefix_lens, suffix_tables=suffix_tables, suffix_lens=suffix_lens,
                        group_ids=group_ids, prefix_parents=prefix_parents),
                   stream=stream, nested=prefix_parents is not None)


def tree_accept(query_offsets, tree_parents, draft_tokens, target_tokens, root_tokens, *, stream=None):
    """One walk on torch int32 tensors; returns (accept_rows, accept_lens, next_tokens)."""
    dev = _device(query_offsets)
    T, R = draft_tokens.shape[0], root_tokens.shape[0]
    with _on_stream(stream, dev):
        rows = make_tree_rows(T, _most_rows(query_offsets), 0, 1)
        taken, lens, follow = (torch.empty(n, dtype=torch.int32, device=dev) for n in (T, R, R))
        parrot_tree_accept(R, rows, query_offsets, tree_parents, draft_tokens, target_tokens, root_tokens, taken, lens,
                           follow, stream=stream)
    return taken, lens, follow


def tree_commit(query_offsets, accept_rows, accept_lens, suffix_k, suffix_v, suffix_tables, suffix_lens, *,
                stream=None):
    """One move in a layer's pools; returns the committed own lengths."""
    with _on_stream(stream, suffix_k.device):
        prob = _cache_problem(suffix_k, suffix_tables, suffix_lens)
        rows = make_tree_rows(accept_rows.shape[0], _most_rows(query_offsets), 0, 1)
        out = torch.empty(accept_lens.shape[0], dtype=torch.int32, device=suffix_k.device)
        parrot_tree_commit(prob, rows, query_offsets, accept_rows, accept_lens, suffix_tables, suffix_lens, suffix_k,
                           suffix_v, out, stream=stream)
    return out
