"""A cache held in 8 bits, as cases that can be timed: fill (norm and rotate the new
rows, write their keys and values in 8 bits with a scale for each block and head),
attend (attention of the new rows over shared prefixes and own tokens in that cache,
for single tokens, drafted chains and prompts), pages (blocks of every layer copied
for forked contexts, or moved together).

A block-head holds 16 tokens.  Codes are e4m3; the scale of a block-head's keys or
values is a power of two (e8m0).  Keys are [block][head][16][D]; values are
[block][head][D / 64][4][16][4][4], token 4 g + t and element 64 x + 4 c + d at
[x][g][c][d][t]; scales are [block][head][2], of the keys and of the values.

Lengths and group structure come from the case alone, so its work is known without a
seed; values and the physical order of the blocks come from the seed.

Fields of a case
  op          fill | attend | pages
  dtype       float32 | float16 | bfloat16, of rows, queries and outputs
  heads       heads of the cache; ratio query heads read each of them
  head_dim
  layers      attend: one plan, then each layer's attention; pages: copied layers
  groups      shared prefixes of prefix_lo .. prefix_hi tokens, read by
              `grouped` requests; ungrouped requests read none
  levels      2: group 0 precedes the others, which add sub_lo .. sub_hi tokens
  own_lo/hi   cached own tokens of a grouped request, free_lo/hi of the others
  rows_lo/hi  new rows per request
  rotary      rotated elements of a head, interleaved or half layout,
              scaling none | linear | ntk | yarn | wavelength by factor
  norm        queries and keys are normalised per head first
  fused       the rows are slices of one projection's output (row strides)
  copies      pages: blocks copied in each pool; wide: the pools hold 16-bit keys and
              values without scales
  lengths     seed of the lengths
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16
MOST = 448.0            # the largest e4m3 value
DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
EPS = 1e-6
BASE = 10000.0
TRAINED = 4096          # positions the scaled rotary frequencies were trained on


def case(name, op, dtype, heads, ratio, head_dim, **kw):
    c = {"op": op, "dtype": dtype, "heads": heads, "ratio": ratio, "head_dim": head_dim, "layers": 1,
         "groups": 0, "grouped": 0, "levels": 1, "prefix_lo": 1, "prefix_hi": 1, "sub_lo": 1,
         "sub_hi": 1, "own_lo": 0, "own_hi": 0, "ungrouped": 0, "free_lo": 0, "free_hi": 0,
         "rows_lo": 1, "rows_hi": 1, "rotary": head_dim, "interleaved": False,
         "scaling": "none", "factor": 1.0, "norm": False, "fused": True, "copies": 0, "wide": False,
         "lengths": 0}
    if name:
        c["name"] = name
    c.update(kw)
    return c


def listed():
    return [
        # a decode step of seven chats: one new row each, where latency counts
        case("fill8_decode_7", "fill", "float16", 32, 1, 128, ungrouped=7, free_lo=40, free_hi=700),
        # a decode step of a large batch, heads normalised, grouped query heads
        case("fill8_decode_256", "fill", "bfloat16", 8, 4, 128, ungrouped=256, free_lo=30, free_hi=900,
             norm=True, interleaved=True),
        # whole prompts of a batch, positions scaled for long contexts
        case("fill8_prompts_12", "fill", "bfloat16", 32, 1, 128, ungrouped=12, rows_lo=100, rows_hi=1500,
             norm=True, scaling="yarn", factor=8.0),
        # the smallest step: four requests on a 128-token prompt
        case("attend8_tiny_f32", "attend", "float32", 4, 1, 64, groups=1, grouped=4, prefix_lo=128,
             prefix_hi=128, own_lo=16, own_hi=200),
        # interactive chats, nothing shared, four layers of a step
        case("attend8_chat_7", "attend", "float16", 32, 1, 128, layers=4, ungrouped=7, free_lo=40, free_hi=700),
        # an ordinary decode batch of a model with grouped query heads, long prompts of their own
        case("attend8_gqa_64", "attend", "bfloat16", 8, 4, 128, layers=2, ungrouped=64, free_lo=500,
             free_hi=6000),
        # a mixed serving step: eight prefixes of many readers, some requests without
        case("attend8_mixed_288", "attend", "bfloat16", 8, 4, 128, layers=2, groups=8, grouped=256, prefix_lo=512,
             prefix_hi=4096, own_lo=32, own_hi=1024, ungrouped=32, free_lo=544, free_hi=5120),
        # a few long conversations, chains of drafted tokens, a query head for each cache head
        case("attend8_long_6", "attend", "float16", 32, 1, 128, ungrouped=6, free_lo=9000, free_hi=33000, rows_lo=3,
             rows_hi=9),
        # a system prompt, few-shot blocks below it, and prompts of many new rows: the largest call
        case("attend8_prompts_12", "attend", "bfloat16", 8, 4, 128, groups=4, grouped=9, levels=2, prefix_lo=4000,
             prefix_hi=4000, sub_lo=300, sub_hi=900, own_lo=0, own_hi=500, ungrouped=3, free_lo=1000, free_hi=3500,
             rows_lo=300, rows_hi=1500),
        # three contexts fork: the partly filled last block of each, over the layers of a model
        case("pages_fork_3", "pages", "float16", 32, 1, 128, layers=16, copies=3),
        # a beam of many contexts forks, grouped query heads
        case("pages_fork_200", "pages", "bfloat16", 8, 4, 128, layers=20, copies=200),
        # a pool of 16-bit blocks is compacted
        case("pages_compact_700", "pages", "float16", 20, 1, 128, layers=6, copies=700, wide=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    while True:
        op = rng.choice(["fill"] * 4 + ["attend"] * 6 + ["pages"] * 2)
        dtype = rng.choice(["float16"] * 4 + ["bfloat16"] * 4 + ["float32"] * 2)
        heads, ratio = rng.choice([(4, 1), (5, 1), (8, 1), (20, 1), (32, 1), (40, 1), (1, 8), (2, 5), (4, 7), (8, 4), (8, 8)])
        dim = rng.choice([128, 128, 128, 64])
        c = case(None, op, dtype, heads, ratio, dim, lengths=rng.randrange(1 << 20))
        prompts = rng.random() < 0.35
        requests = _log_int(rng, 1, 32 if prompts else 256)
        c["ungrouped"] = requests
        c["rows_lo"] = _log_int(rng, 1, 500) if prompts else rng.choice([1, 1, 1, _log_int(rng, 1, 32)])
        c["rows_hi"] = c["rows_lo"] + (0 if rng.random() < 0.5 else _log_int(rng, 1, 1500 if prompts else 16))
        c["free_lo"] = 0 if prompts and rng.random() < 0.5 else _log_int(rng, 1, 1500)
        c["free_hi"] = c["free_lo"] + _log_int(rng, 1, 1500)
        if op == "fill":
            c["rotary"] = rng.choice([dim, dim, dim, dim // 2, dim // 4, 20, 50])
            c["interleaved"] = rng.random() < 0.4
            c["scaling"] = rng.choice(["none", "none", "linear", "ntk", "yarn", "wavelength"])
            c["factor"] = 1.0 if c["scaling"] == "none" else rng.choice([2.0, 4.0, 8.0, 32.0])
            c["norm"] = rng.random() < 0.5
            c["fused"] = rng.random() < 0.7
        if op == "attend":
            c["layers"] = rng.choice([1, 1, 2, 4])
            if not prompts:
                c["free_lo"] = _log_int(rng, 1, 20000)
                c["free_hi"] = c["free_lo"] + _log_int(rng, 1, 13000)
            if rng.random() < 0.7 and requests > 1:
                c["ungrouped"] = rng.randint(0, requests // 4)
                c["grouped"] = requests - c["ungrouped"]
                c["groups"] = _log_int(rng, 1, max(1, min(16, c["grouped"])))
                c["levels"] = rng.choice([1, 1, 2])
                c["groups"] = max(c["groups"], c["levels"])
                c["prefix_lo"] = _log_int(rng, 16, 3000)
                c["prefix_hi"] = c["prefix_lo"] + (0 if rng.random() < 0.4 else _log_int(rng, 1, 4000))
                c["sub_lo"] = _log_int(rng, 1, 300)
                c["sub_hi"] = c["sub_lo"] + _log_int(rng, 1, 400)
                c["own_lo"] = rng.choice([0, _log_int(rng, 1, 200)])
                c["own_hi"] = c["own_lo"] + _log_int(rng, 1, 1000)
        if op == "pages":
            c["layers"] = _log_int(rng, 1, 20)
            c["copies"] = _log_int(rng, 1, 1500)
            c["wide"] = rng.random() < 0.3
        w = work(c)
        most = {"fill": 5.0e8, "attend": 1.0e9, "pages": 1.0e9}[op]
        most_flops = 8.0e11 if dtype != "float32" else 1.0e11
        if w["bytes"] > most or w["flops"] > most_flops:
            continue
        if op == "attend":
            # the plain form attends to keys padded to the longest context
            at = layout(c)
            n, rows = len(at["own"]), int(at["rows"].max())
            keys = c["levels"] * int(at["plen"].max(initial=0)) + int(at["own"].max())
            if n * keys * heads * dim > 6.0e9 or n * keys * heads * ratio * rows > 1.2e10:
                continue
            if int(at["own"].sum()) * heads * dim * c["layers"] > 8.0e8:
                continue
        return c


# ------------------------------------------------------------------- layout
def _chain(g, parents):
    return [] if g < 0 else _chain(parents[g], parents) + [g]


def layout(c):
    """Lengths and groups of a case (host arrays)."""
    rng = np.random.default_rng([c["lengths"], c["grouped"], c["ungrouped"], c["rows_hi"]])
    ng, n = c["groups"], c["grouped"] + c["ungrouped"]
    first = 1 if c["levels"] > 1 else 0
    plen = rng.integers(c["prefix_lo"], c["prefix_hi"] + 1, ng)
    if first:
        plen[1:] = rng.integers(c["sub_lo"], c["sub_hi"] + 1, ng - 1)
    parents = np.array([-1] * first + [0 if first else -1] * (ng - first), dtype=np.int64)
    gid = np.concatenate([first + np.arange(c["grouped"]) % max(1, ng - first),
                          np.full(c["ungrouped"], -1)]).astype(np.int64)
    cached = np.concatenate([rng.integers(c["own_lo"], c["own_hi"] + 1, c["grouped"]),
                             rng.integers(c["free_lo"], c["free_hi"] + 1, c["ungrouped"])])
    rows = rng.integers(c["rows_lo"], c["rows_hi"] + 1, n)
    shuffled = rng.permutation(n)
    gid, cached, rows = gid[shuffled], cached[shuffled], rows[shuffled]
    before = np.array([sum(plen[a] for a in _chain(g, parents)) for g in gid], dtype=np.int64)
    return {"gid": gid, "plen": plen, "parents": parents, "cached": cached, "rows": rows, "own": cached + rows,
            "off": np.concatenate([[0], np.cumsum(rows)]), "before": before}


def work(c):
    """What each operator cannot do without (each input and output once)."""
    elt = 4 if c["dtype"] == "float32" else 2
    h, d = c["heads"], c["head_dim"]
    if c["op"] == "pages":
        block = 2 * h * BLOCK * d * elt if c["wide"] else 2 * h * (BLOCK * d + 1)
        return {"bytes": 2 * c["copies"] * c["layers"] * block + 8 * c["copies"], "flops": 0}
    at = layout(c)
    total = int(at["off"][-1])
    wide = h * d * elt                                           # K or V of one row
    if c["op"] == "fill":
        return {"bytes": total * (2 * wide * (c["ratio"] + 1) + 2 * h * d + 4),
                "flops": total * h * ((c["ratio"] + 1) * (3 * c["rotary"] + (4 * d if c["norm"] else 0)) + 4 * d)}
    read = {a for g in at["gid"] for a in _chain(g, at["parents"])}
    tokens = int(sum(at["plen"][g] for g in read)) + int(at["own"].sum())
    blocks = int(sum(-(-at["plen"][g] // BLOCK) for g in read)) + int((-(-at["own"] // BLOCK)).sum())
    rows, seen = at["rows"], at["before"] + at["cached"]
    keys = int(np.sum(rows * seen + rows * (rows + 1) // 2))
    hq = h * c["ratio"]
    return {"bytes": c["layers"] * (2 * tokens * h * d + 2 * blocks * h + 2 * total * hq * d * elt + 4 * total * hq),
            "flops": c["layers"] * 4 * keys * hq * d}


# -------------------------------------------------------------------- inputs
def _need(most):
    """The exponent byte of the smallest power of two that takes `most` to at most 448."""
    mantissa, power = torch.frexp(most)
    return torch.where(most > 0, (power - 9 + (mantissa > MOST / 512).int() + 127).clamp(1, 254), 0)


def _encode(y, byte):
    """e4m3 codes of y / 2^(byte - 127), as bytes."""
    y = torch.where(y.isfinite(), torch.ldexp(y, 127 - byte), math.nan)
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _value_order(x):
    """[.., 16, D] as the values' blocks hold it."""
    x = x.unflatten(-1, (-1, 16, 4)).unflatten(-4, (4, 4))       # g t x c d
    return x.movedim((-3, -5, -2, -1, -4), (-5, -4, -3, -2, -1))  # x g c d t


def _token_order(x):
    """A value block as [.., 16, D]."""
    x = x.movedim((-4, -1, -5, -3, -2), (-5, -4, -3, -2, -1))    # x g c d t -> g t x c d
    return x.flatten(-3).flatten(-3, -2)


def _packed(dense):
    """Codes and scale bytes of blocks [n, H, 16, D]."""
    byte = _need(dense.abs().amax((2, 3)).float())
    return _encode(dense.float(), byte[..., None, None]), byte


def _pools(n, h, d, draw_block):
    """Keys, values and scales of n blocks, as the framework holds them."""
    step = max(1, (1 << 26) // (h * BLOCK * d))
    parts = [(_packed(draw_block(min(step, n - i), 0)), _packed(draw_block(min(step, n - i), 1))) for i in range(0, n, step)]
    return {"k": torch.cat([k for (k, _), _ in parts]).view(torch.float8_e4m3fn),
            "v": torch.cat([_value_order(v) for _, (v, _) in parts]).contiguous().view(torch.float8_e4m3fn),
            "scales": torch.cat([torch.stack([a, b], -1) for (_, a), (_, b) in parts]).to(torch.uint8).view(torch.float8_e8m0fnu)}


def prepare(c, seed):
    host = np.random.default_rng([int(seed), 91])
    dev = torch.device("cuda")
    h, hq, d, dt = c["heads"], c["heads"] * c["ratio"], c["head_dim"], DTYPES[c["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 6151 + 29)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev, dtype=dt)

    def ints(x):
        return torch.tensor(np.asarray(x, dtype=np.int32), device=dev)

    if c["op"] == "pages":
        n, held = c["copies"], 2 * c["copies"] + 5
        ids = host.permutation(held)
        if c["wide"]:
            pools = [normal(held, h, BLOCK, d) for _ in range(2 * c["layers"])]
        else:
            code = lambda *shape: torch.randint(0, 127, shape, generator=gen, device=dev, dtype=torch.uint8)
            each = [(code(held, h, BLOCK, d).view(torch.float8_e4m3fn),
                     code(held, h, d // 64, 4, 16, 4, 4).view(torch.float8_e4m3fn),
                     code(held, h, 2).add_(60).view(torch.float8_e8m0fnu)) for _ in range(c["layers"])]
            pools = [x for layer in each for x in layer]
        return {"case": c, "pools": pools, "src": ints(ids[:n]), "dst": ints(ids[n:2 * n])}

    at = layout(c)
    n, total = len(at["rows"]), int(at["off"][-1])
    # keys and values of the heads differ in size
    loud = torch.rand(2, h, 1, 1, generator=gen, device=dev).mul_(3).sub_(1.5).exp2_()

    def blocks(m, which):
        return torch.randn(m, h, BLOCK, d, generator=gen, device=dev) * loud[which]

    def tables(lens):
        need = [-(-int(x) // BLOCK) for x in lens]
        ids = host.permutation(sum(need)).astype(np.int32)
        t = np.zeros((len(lens), max(need + [1])), dtype=np.int32)
        start = 0
        for i, k in enumerate(need):
            t[i, :k] = ids[start:start + k]
            start += k
        return t, max(sum(need), 1)

    stab, nown = tables(at["own"])
    t = {"query_offsets": ints(at["off"]), "suffix_tables": ints(stab), "suffix_lens": ints(at["own"])}
    if c["op"] == "fill":
        t["suffix"] = _pools(nown, h, d, blocks)
        if c["fused"]:
            x = normal(total, (hq + 2 * h) * d)
            t["q_rows"], t["k_rows"], t["v_rows"] = (
                y.unflatten(1, (-1, d)) for y in x.split([hq * d, h * d, h * d], 1))
        else:
            t["q_rows"], t["k_rows"], t["v_rows"] = normal(total, hq, d), normal(total, h, d), normal(total, h, d)
        if c["norm"]:
            t["q_norm"], t["k_norm"] = 1 + 0.1 * normal(d), 1 + 0.1 * normal(d)
        place = np.arange(total) - np.repeat(at["off"][:-1], at["rows"])
        t["positions"] = ints(np.repeat(at["before"] + at["cached"], at["rows"]) + place)
    else:
        ptab, npre = tables(at["plen"])
        t["prefix_tables"], t["prefix_lens"] = ints(ptab), ints(at["plen"])
        t["prefix_parents"], t["group_ids"] = ints(at["parents"]), ints(at["gid"])
        t["layers"] = [{"q_rows": normal(total, hq, d), "prefix": _pools(npre, h, d, blocks),
                        "suffix": _pools(nown, h, d, blocks)} for _ in range(c["layers"])]
    # sizes that an engine keeps on the host beside the device arrays
    sizes = {"at": at, "nown": nown, "most": int(at["rows"].max()), "longest": int(at["own"].max()),
             "longest_prefix": int(at["plen"].max()) if c["groups"] else 0}
    return {"case": c, "t": t, "sizes": sizes}


# ------------------------------------------------------ the framework's calls
def _bind(state):
    """The handles that an engine makes once for a batch: the calls and their results."""
    import paper_2405_19888_amd as parrot
    c = state["case"]
    if c["op"] == "pages":
        copier = parrot.BlockCopier(state["pools"], c["copies"])
        return [copier.bind(state["src"], state["dst"])], state["pools"]
    t, s = state["t"], state["sizes"]
    at, d = s["at"], c["head_dim"]
    attend = c["op"] == "attend"
    nested = attend and c["levels"] > 1
    prob = parrot.problem_from_host(
        num_heads=c["heads"], head_dim=d, block_size=BLOCK, dtype=DTYPES[c["dtype"]], sm_scale=d ** -0.5,
        group_ids=at["gid"] if attend else [-1] * len(at["gid"]), prefix_lens=at["plen"] if attend else [],
        suffix_lens=at["own"], prefix_table_stride=t["prefix_tables"].shape[1] if attend else 0,
        suffix_table_stride=t["suffix_tables"].shape[1], num_suffix_blocks=s["nown"],
        num_prefix_blocks=t["layers"][0]["prefix"]["k"].shape[0] if attend else 0,
        prefix_parents=at["parents"] if nested else None)
    if c["op"] == "fill":
        scale = {} if c["scaling"] == "none" else {"scaling": c["scaling"], "factor": c["factor"], "original_length": TRAINED}
        rotary = parrot.make_rotary(c["rotary"], base=BASE, interleaved=c["interleaved"], **scale)
        fill = parrot.Cache8Filler(prob, int(at["off"][-1]), s["most"], c["heads"] * c["ratio"], rotary=rotary, norm_eps=EPS)
        return [fill.bind(t)], {"q": fill.q_out, **t["suffix"]}
    rows = parrot.tree_rows_from_host(at["off"], at["gid"], c["groups"], c["heads"] * c["ratio"],
                                      at["parents"] if nested else None)
    plan = parrot.Cache8Planner(prob, rows, nested=nested)
    each = [parrot.Cache8Decoder(plan) for _ in t["layers"]]
    return ([plan.bind(t)] + [dec.bind({**t, **x}) for dec, x in zip(each, t["layers"])],
            [{"out": dec.out, "lse": dec.lse} for dec in each])


# ----------------------------------------------------------- the plain forms
def _requests(t):
    """Each row's request and its place among the request's rows."""
    off = t["query_offsets"].long()
    row = torch.arange(t["total"], device=off.device)
    request = torch.searchsorted(off, row, right=True) - 1
    return request, row - off[request]


def _frequencies(c):
    half = c["rotary"] // 2
    i = torch.arange(half, dtype=torch.float64)
    base = BASE * c["factor"] ** (c["rotary"] / (c["rotary"] - 2)) if c["scaling"] == "ntk" else BASE
    f = base ** (-2 * i / c["rotary"])
    if c["scaling"] == "linear":
        return f / c["factor"], 1.0
    if c["scaling"] == "yarn":
        place = lambda turns: c["rotary"] * math.log(TRAINED / (turns * 2 * math.pi)) / (2 * math.log(BASE))
        lo, hi = max(math.floor(place(32.0)), 0), min(math.ceil(place(1.0)), c["rotary"] - 1)
        kept = 1 - ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f * (kept + (1 - kept) / c["factor"]), 0.1 * math.log(c["factor"]) + 1.0
    if c["scaling"] == "wavelength":
        kept = ((TRAINED * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f * (kept + (1 - kept) / c["factor"]), 1.0
    return f, 1.0


def _rotated(c, x, weight, positions):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    f, amplitude = _frequencies(c)
    angle = positions.double()[:, None, None] * f.to(x.device)
    cos, sin = (angle.cos() * amplitude).float(), (angle.sin() * amplitude).float()
    turned, rest = x[..., :c["rotary"]], x[..., c["rotary"]:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if c["interleaved"] else turned.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, rest], -1)


def _written(rows, unit, offset, fresh, codes, byte):
    """The blocks' new codes [U, H, 16, D] and bytes [U, H]: rows [T, H, D] go to `offset` of
    block `unit`; the slots before a block's first row are kept unless it is fresh."""
    new = torch.zeros(*codes.shape, device=codes.device)
    new[unit, :, offset] = rows
    size = torch.zeros(byte.shape[0], BLOCK, byte.shape[1], device=codes.device)
    size[unit, offset] = torch.where(rows.isfinite(), rows, 0).abs().amax(-1)
    need = _need(size.amax(1))
    now = torch.where(fresh[:, None], need, torch.maximum(need, byte.int()))
    written = torch.zeros(byte.shape[0], BLOCK, dtype=torch.bool, device=codes.device)
    written[unit, offset] = True
    first = written.int().argmax(1)
    kept = (torch.arange(BLOCK, device=codes.device) < first[:, None])[:, None, :, None]
    moved = torch.ldexp(codes.view(torch.float8_e4m3fn).float(), (byte.int() - now)[..., None, None])
    moved = torch.where((now > byte.int())[..., None, None], moved.to(torch.float8_e4m3fn).view(torch.uint8), codes)
    out = torch.where(written[:, None, :, None], _encode(new, now[..., None, None]), torch.where(kept, moved, codes))
    return out, now.to(torch.uint8)


def _plain_fill(c, t):
    dt = DTYPES[c["dtype"]]
    t = {**t, "total": t["positions"].shape[0]}
    request, place = _requests(t)
    cached = t["suffix_lens"].long() - t["query_offsets"].long().diff()
    position = cached[request] + place
    block = t["suffix_tables"].long()[request, position // BLOCK]
    touched, unit = block.unique(return_inverse=True)
    fresh = torch.zeros(touched.shape[0], dtype=torch.bool, device=block.device)
    fresh[unit[position % BLOCK == 0]] = True
    k, v, scales = (t["suffix"][x].view(torch.uint8) for x in ("k", "v", "scales"))
    codes, byte = _written(_rotated(c, t["k_rows"], t.get("k_norm"), t["positions"]), unit, position % BLOCK, fresh,
                           k[touched], scales[touched, :, 0])
    k[touched], scales[touched, :, 0] = codes, byte
    codes, byte = _written(t["v_rows"].float(), unit, position % BLOCK, fresh, _token_order(v[touched]),
                           scales[touched, :, 1])
    v[touched], scales[touched, :, 1] = _value_order(codes), byte
    return {"q": _rotated(c, t["q_rows"], t.get("q_norm"), t["positions"]).to(dt), **t["suffix"]}


def _dense(pool, which, table):
    """Keys or values [n, H, tokens, D] of tables [n, blocks], as the values they stand for."""
    codes = pool["kv"[which]].view(torch.uint8)[table].view(torch.float8_e4m3fn).float()
    codes = _token_order(codes) if which else codes
    size = pool["scales"].view(torch.uint8)[table][..., which].int() - 127               # [n, blocks, H]
    return torch.ldexp(codes, size[..., None, None]).transpose(1, 2).flatten(2, 3)


def _plain_attend(c, t, layer, sizes):
    h, ratio, d, dt = c["heads"], c["ratio"], c["head_dim"], DTYPES[c["dtype"]]
    most, longest, n = sizes["most"], sizes["longest"], t["suffix_lens"].shape[0]
    request, place = _requests({**t, "total": layer["q_rows"].shape[0]})
    dev = request.device
    q = torch.zeros(n, most, h, ratio, d, device=dev)
    q[request, place] = layer["q_rows"].float().unflatten(1, (h, ratio))
    # keys: the chain's prefixes, innermost first, then the own tokens
    blocks = lambda k: -(-k // BLOCK)
    chain = [t["group_ids"].long()]
    if c["levels"] > 1:
        chain.append(torch.where(chain[0] >= 0, t["prefix_parents"].long()[chain[0].clamp(min=0)], -1))
    held = [t["prefix_tables"].long()[g.clamp(min=0), :blocks(sizes["longest_prefix"])] for g in chain if c["groups"]]
    mine = t["suffix_tables"].long()[:, :blocks(longest)]
    k = torch.cat([_dense(layer["prefix"], 0, x) for x in held] + [_dense(layer["suffix"], 0, mine)], 2)
    v = torch.cat([_dense(layer["prefix"], 1, x) for x in held] + [_dense(layer["suffix"], 1, mine)], 2)
    # what each row sees
    count = lambda table: torch.arange(table.shape[1] * BLOCK, device=dev)
    seen = [((g >= 0)[:, None] & (count(x) < t["prefix_lens"].long()[g.clamp(min=0)][:, None]))[:, None].expand(-1, most, -1)
            for g, x in zip(chain, held)]
    cached = t["suffix_lens"].long() - t["query_offsets"].long().diff()
    position = cached[:, None] + torch.arange(most, device=dev)                          # [n, most]
    seen.append(count(mine) <= position[..., None])
    seen = torch.cat(seen, 2)                                                            # [n, most, keys]
    right = q.permute(0, 2, 4, 1, 3).reshape(n, h, d, most * ratio).contiguous()
    x = torch.matmul(k, right).mul_(d ** -0.5).unflatten(3, (most, ratio))               # [n, H, keys, most, ratio]
    x = x.masked_fill_(~seen.transpose(1, 2)[:, None, :, :, None], -math.inf)
    top = x.amax(2, keepdim=True)
    top = torch.where(top.isfinite(), top, 0)
    x = x.sub_(top).exp_()
    total = x.sum(2)                                                                     # [n, H, most, ratio]
    out = torch.matmul(x.flatten(3).transpose(2, 3), v).unflatten(2, (most, ratio))      # [n, H, most, ratio, D]
    out = (out / total[..., None]).permute(0, 2, 1, 3, 4)[request, place].flatten(1, 2)
    lse = (top[:, :, 0] + total.log()).permute(0, 2, 1, 3)[request, place].flatten(1, 2)
    return {"out": out.to(dt), "lse": lse}


def _plain_copy(pool, src, dst):
    pool = pool.view(torch.uint8) if pool.dtype.itemsize == 1 else pool
    pool[dst] = pool[src]


def run(state):
    c = state["case"]
    if own:
        if "calls" not in state:
            state["calls"], state["results"] = _bind(state)
        [call() for call in state["calls"]]
        return state["results"]
    if c["op"] == "pages":
        src, dst = state["src"].long(), state["dst"].long()
        [_plain_copy(pool, src, dst) for pool in state["pools"]]
        return state["pools"]
    if c["op"] == "fill":
        return _plain_fill(c, state["t"])
    return [_plain_attend(c, state["t"], layer, state["sizes"]) for layer in state["t"]["layers"]]


# --------------------------------------------------------------- the results
def _exact_codes(y, power):
    """e4m3 values nearest to y / 2^power, ties to even, in 64 bits."""
    x = y * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=y.device), -power.double())
    size = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -60)))
    size = torch.where(2.0 ** size > x.abs(), size - 1, size).clamp(min=-6)              # (log2 rounds up to whole numbers)
    size = torch.where(2.0 ** (size + 1) <= x.abs(), size + 1, size)
    step = 2.0 ** (size - 3)
    return torch.round(x / step) * step


def _exact_power(most):
    """The least whole power with most / 2^power <= 448 (-127: nothing but zeros)."""
    power = torch.ceil(torch.log2(most.clamp(min=2.0 ** -140) / MOST))
    power = torch.where(most > MOST * 2.0 ** power, power + 1, power)
    power = torch.where(most <= MOST * 2.0 ** (power - 1), power - 1, power)
    return torch.where(most > 0, power.clamp(min=-126), -127)


def exact(c, seed):
    """The same outputs request by request, in 64 bits and on the host's indices."""
    state = prepare(c, seed)
    if c["op"] == "pages":
        src, dst = state["src"].tolist(), state["dst"].tolist()
        at = list(range(state["pools"][0].shape[0]))
        for a, b in zip(src, dst):
            at[b] = a
        at = torch.tensor(at, device="cuda")
        whole = lambda x: (x.view(torch.uint8)[at].view(x.dtype) if x.dtype.itemsize == 1 else x[at]).float().double()
        return [whole(x) for x in state["pools"]]
    t, at = state["t"], state["sizes"]["at"]
    stab = t["suffix_tables"].cpu().numpy()
    h, ratio, d = c["heads"], c["ratio"], c["head_dim"]
    n = len(at["rows"])
    token = torch.arange(BLOCK)[:, None]
    element = torch.arange(d)[None]
    # where [token, element] of a value block is
    where = ((((element // 64 * 4 + token // 4) * 16 + element % 64 // 4) * 4 + element % 4) * 4 + token % 4).cuda()

    def values(pool, which, ids):        # [blocks, H, 16, D] in 64 bits, and the powers
        ids = torch.as_tensor(np.asarray(ids), device="cuda").long()
        code = pool["kv"[which]].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float().double().flatten(2)
        code = code[:, :, where] if which else code.unflatten(2, (BLOCK, d))
        return code, pool["scales"].view(torch.uint8)[ids, :, which].double() - 127

    if c["op"] == "fill":
        rd, s = c["rotary"], c["factor"]
        radians, amplitude = [], 1.0
        for i in range(rd // 2):
            x = BASE ** (-2.0 * i / rd)
            if c["scaling"] == "linear":
                x /= s
            elif c["scaling"] == "ntk":
                x = (BASE * s ** (rd / (rd - 2.0))) ** (-2.0 * i / rd)
            elif c["scaling"] == "yarn":
                at_turns = lambda k: rd / 2.0 * (math.log(TRAINED) - math.log(2.0 * math.pi * k)) / math.log(BASE)
                lo, hi = max(0, math.floor(at_turns(32))), min(rd - 1, math.ceil(at_turns(1)))
                blend = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
                x = x * (1.0 - blend) + x / s * blend
                amplitude = 1.0 + math.log(s) / 10.0
            elif c["scaling"] == "wavelength":
                turns = TRAINED * x / (2.0 * math.pi)
                blend = min(1.0, max(0.0, (4.0 - turns) / 3.0))
                x = x * (1.0 - blend) + x / s * blend
            radians.append(x)
        angle = t["positions"].double()[:, None] * torch.tensor(radians, dtype=torch.float64, device="cuda")[None]
        turn = torch.polar(torch.full_like(angle, amplitude), angle)[:, None]            # [T, 1, pairs]

        def rotated(x, weight):
            x = x.double()
            if c["norm"]:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS) * weight.double()
            one = list(range(0, rd, 2)) if c["interleaved"] else list(range(rd // 2))
            two = [i + 1 for i in one] if c["interleaved"] else [i + rd // 2 for i in one]
            y = torch.complex(x[..., one].contiguous(), x[..., two].contiguous()) * turn
            x = x.clone()
            x[..., one], x[..., two] = y.real, y.imag
            return x

        new = [rotated(t["k_rows"], t.get("k_norm")), t["v_rows"].double()]
        # the blocks that rows go to: block id, first slot, rows
        jobs = []
        for r in range(n):
            p, end, row = int(at["cached"][r]), int(at["own"][r]), int(at["off"][r])
            while p < end:
                m = min(end - p, BLOCK - p % BLOCK)
                jobs.append((int(stab[r, p // BLOCK]), p % BLOCK, m, row))
                p, row = p + m, row + m
        job = np.array(jobs)
        slot = torch.arange(BLOCK, device="cuda")[None]
        first, count, row = (torch.as_tensor(job[:, i], device="cuda")[:, None] for i in (1, 2, 3))
        fresh = first == 0
        mine = (slot >= first) & (slot < first + count)                                  # [jobs, 16]
        source = (row + slot - first).clamp(0, new[0].shape[0] - 1)
        result = {"q": rotated(t["q_rows"], t.get("q_norm"))}
        powers = []
        for which in (0, 1):
            code, power = values(t["suffix"], which, job[:, 0])
            x = new[which][source].transpose(1, 2) * mine[:, None, :, None]              # [jobs, H, 16, D]
            need = _exact_power(x.abs().amax((2, 3)))
            now = torch.where(fresh, need, torch.maximum(need, power))
            raised = (now > power)[..., None, None]
            again = _exact_codes(code, (now - power)[..., None, None])
            kept = torch.where(raised & (slot < first)[:, None, :, None], again, code)
            code = torch.where(mine[:, None, :, None], _exact_codes(x, now[..., None, None]), kept)
            pool = t["suffix"]["kv"[which]].float().double()
            ids = torch.as_tensor(job[:, 0], device="cuda")
            if which:
                flat = torch.empty(*code.shape[:2], BLOCK * d, dtype=torch.float64, device="cuda")
                flat[:, :, where.flatten()] = code.flatten(2)
                code = flat.view(-1, *pool.shape[1:])
            pool[ids] = code
            result["kv"[which]] = pool
            powers.append(now)
        sizes = t["suffix"]["scales"].float().double()
        sizes[torch.as_tensor(job[:, 0], device="cuda")] = 2.0 ** torch.stack(powers, -1)
        return {**result, "scales": sizes}

    ptab = t["prefix_tables"].cpu().numpy()

    def tokens(pool, which, table, count):      # [H, count, D] in 64 bits
        code, power = values(pool, which, table[: -(-count // BLOCK)])
        return (code * (2.0 ** power)[..., None, None]).transpose(0, 1).reshape(h, -1, d)[:, :count]

    results = []
    for layer in t["layers"]:
        out = torch.empty(layer["q_rows"].shape, dtype=torch.float64, device="cuda")
        lse = torch.empty(layer["q_rows"].shape[:2], dtype=torch.float64, device="cuda")
        for r in range(n):
            o, e, before = int(at["off"][r]), int(at["off"][r + 1]), int(at["before"][r]) + int(at["cached"][r])
            parts = [(layer["prefix"], ptab[g], int(at["plen"][g])) for g in _chain(int(at["gid"][r]), at["parents"])]
            parts.append((layer["suffix"], stab[r], int(at["own"][r])))
            k, v = (torch.cat([tokens(pool, which, tab, m) for pool, tab, m in parts if m], 1).contiguous() for which in (0, 1))
            kt = k.transpose(1, 2).contiguous()
            hidden = torch.arange(k.shape[1], device="cuda")[None] > before + torch.arange(e - o, device="cuda")[:, None]
            for g in range(ratio):
                x = torch.matmul(layer["q_rows"][o:e, g::ratio].double().transpose(0, 1).contiguous(), kt) * d ** -0.5
                x = x.masked_fill(hidden[None], -math.inf)
                total = torch.logsumexp(x, -1)
                out[o:e, g::ratio] = torch.matmul(torch.exp(x - total[..., None]), v).transpose(0, 1)
                lse[o:e, g::ratio] = total.transpose(0, 1)
        results.append({"out": out, "lse": lse})
    return results
