"""A batch that answers with samples over a cache held in 4 bits: its operators as cases that can be timed, each in a plain form and as a
call of the framework.

  append   new positions rotated, their keys and values put into 4-bit KV tiles, and read back as bf16
  attn     attention of new queries over 4-bit KV tiles: single tokens, a few drafted tokens, prompts
  move     sequences of a batch copied, forked, compacted and freed inside the KV tiles, bf16 or 4-bit
  sample   the next token of every sequence by temperature, top-k, top-p and min-p from a given random number

A KV tile in 4 bits holds TK positions of B sequences and Hkv heads.  A page (one sequence, one head of it) is TK rows of Dh / 2 bytes, two
e2m1 numbers per byte with the lower dimension in the lower half, and behind them TK rows of Dh / 16 scales in e4m3, one for 16 dimensions.
An element stands for code * scale * 2^exp, the exponent being the layer's, one for keys and one for values.

Head counts, dimensions, tile sizes and vocabularies are those of the repository's configurations or generic ones.
"""
import math

import numpy as np
import torch

own = False

SMALL = dict(Hq=32, Hkv=8, Dh=64)              # heads of a 1B decoder
MEDIUM = dict(Hq=32, Hkv=8, Dh=128)            # heads of an 8B decoder
LARGE = dict(Hq=64, Hkv=8, Dh=128)             # heads of a 70B decoder


def listed():
    return [
        # a decode step of eight users: the new token of each goes into the cache
        dict(MEDIUM, name="append_decode_b8", op="append", B=8, S=1, pos0=1279, TK=256, ragged=False, k_exp=0, v_exp=-2),
        # the prompts of four users on a large model
        dict(LARGE, name="append_prefill_8k", op="append", B=4, S=2048, pos0=0, TK=64, ragged=False, k_exp=0, v_exp=-2),
        # one user, one token, a short cache: nothing but latency
        dict(SMALL, name="attn_decode_b1", op="attn", B=1, S=1, pos0=700, TK=128, ragged=False, k_exp=0, v_exp=-2),
        # a busy server's step: users at positions of their own, some places of the batch idle
        dict(MEDIUM, name="attn_decode_ragged_b61", op="attn", B=61, S=1, pos0=2500, TK=128, ragged=True, k_exp=1, v_exp=-2),
        # 24 users far into long documents: the cache does not fit L2 even in 4 bits
        dict(LARGE, name="attn_decode_long_b24", op="attn", B=24, S=1, pos0=12000, TK=256, ragged=False, k_exp=0, v_exp=-2),
        # five drafted tokens of three users are verified at once
        dict(MEDIUM, name="attn_verify_b3", op="attn", B=3, S=5, pos0=2000, TK=256, ragged=False, k_exp=0, v_exp=0),
        # a chunk of prompt behind 1500 cached positions, sizes that fit no tile
        dict(MEDIUM, name="attn_chunk_b3", op="attn", B=3, S=201, pos0=1500, TK=256, ragged=False, k_exp=0, v_exp=-2),
        # whole prompts on a large model
        dict(LARGE, name="attn_prefill_b2", op="attn", B=2, S=2048, pos0=0, TK=64, ragged=False, k_exp=0, v_exp=-2),
        # one prompt becomes sixteen answers, before the first of their tokens (bf16 tiles)
        dict(MEDIUM, name="move_fork_b16", op="move", form="bf16", kind="fork", B=16, len=2111, TK=64),
        # a third of a batch has finished: sequences from the end take the free places (4-bit tiles)
        dict(MEDIUM, name="move_compact_b61", op="move", form="q4", kind="compact", B=61, len=700, TK=128),
        # one user, every filter
        dict(name="sample_b1", op="sample", B=1, V=32000, filters="all"),
        # a server's step: users with settings of their own over a large vocabulary
        dict(name="sample_b64", op="sample", B=64, V=128256, filters="mixed"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """A case of the same ranges: one to 96 sequences, caches of one to 16000 positions, vocabularies of some thousands to 128256."""
    op = rng.choice(["append", "attn", "attn", "attn", "attn", "move", "sample", "sample"])
    if op == "sample":
        V = _log_int(rng, 4001, 128256)
        return dict(op=op, B=_log_int(rng, 1, min(96, 8_000_000 // V)), V=V, filters=rng.choice(["none", "top_k", "top_p", "min_p", "all", "mixed"]))
    Dh, Hkv, group = rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 8])
    heads = dict(Hq=Hkv * group, Hkv=Hkv, Dh=Dh)
    if op == "move":
        B = _log_int(rng, 3, 96)
        n = _log_int(rng, 1, min(8000, 100_000_000 // (B * Hkv * Dh)))
        return dict(heads, op=op, form=rng.choice(["bf16", "q4"]), kind=rng.choice(["fork", "compact", "free"]), B=B, len=n, TK=_tile(rng, n))
    exps = dict(k_exp=rng.choice([0, 0, 1, -3]), v_exp=rng.choice([0, -2, -2, 2]))
    kind = rng.choice(["decode", "decode", "decode", "few", "prefill"])
    if kind == "decode":
        B = _log_int(rng, 1, 96)
        pos0 = _log_int(rng, 1, min(16000, 250_000_000 // (B * Hkv * Dh))) - 1
        return dict(heads, **exps, op=op, B=B, S=1, pos0=pos0, TK=_tile(rng, pos0 + 1), ragged=rng.random() < 0.4)
    if kind == "few":
        B, S = _log_int(rng, 1, 16), _log_int(rng, 2, 100)
        pos0 = rng.choice([0, _log_int(rng, 1, min(8000, 60_000_000 // (B * Hkv * Dh)))])
        return dict(heads, **exps, op=op, B=B, S=S, pos0=pos0, TK=_tile(rng, pos0 + S), ragged=False)
    B = _log_int(rng, 1, 8)
    S = _log_int(rng, 100, 4000 // B)
    pos0 = rng.choice([0, _log_int(rng, 1, 2000)])
    return dict(heads, **exps, op=op, B=B, S=S, pos0=pos0, TK=_tile(rng, pos0 + S), ragged=False)


def _tile(rng, n):
    """Positions per KV tile, of which a call addresses 64 at most."""
    return rng.choice([t for t in (16, 32, 64, 128, 256) if 64 * t >= n])


# ---- what a case says besides its sizes -----------------------------------------------------------------------------------------

def _positions(case):
    """The position of each sequence's new token; -1 where a place of the batch is idle."""
    at = np.arange(case["B"])
    pos = np.floor((at * 0.6180339887 % 1.0) * case["pos0"] + 0.5)
    pos[0] = case["pos0"]
    return np.where(at % 9 == 4, -1, pos).astype(np.int32)


def _pairs(case):
    """Which sequence goes where: (from, to), from -1 where a place is freed."""
    B = case["B"]
    if case["kind"] == "fork":
        return [(0, b) for b in range(1, B)]
    gone = [b for b in range(B) if b % 3 == 1]
    if case["kind"] == "free":
        return [(-1, b) for b in gone]
    live = B - len(gone)
    return list(zip([b for b in range(live, B) if b % 3 != 1], [b for b in gone if b < live]))


def _row_bytes(case):
    """Bytes of one position of one head of a tile."""
    return case["Dh"] * 2 if case.get("form") == "bf16" else case["Dh"] // 2 + case["Dh"] // 16


def work(case):
    c = case
    if c["op"] == "sample":
        return dict(bytes=4 * c["B"] * c["V"] + 8 * c["B"], flops=2 * c["B"] * c["V"])
    if c["op"] == "move":
        pairs, page = _pairs(c), 2 * c["Hkv"] * c["len"] * _row_bytes(c)
        return dict(bytes=page * (len({a for a, _ in pairs if a >= 0}) + len(pairs)), flops=0)
    qd, kd = c["Hq"] * c["Dh"], c["Hkv"] * c["Dh"]
    cached, M = 2 * c["Hkv"] * _row_bytes(c), c["B"] * c["S"]
    if c["op"] == "append":
        return dict(bytes=M * (6 * qd + 8 * kd + cached + 4 * kd) + 4 * c["S"] * c["Dh"], flops=6 * M * (qd + 2 * kd))
    if c["ragged"]:
        keys = pairs = int(np.sum(_positions(c) + 1))
    else:
        keys, pairs = c["B"] * (c["pos0"] + c["S"]), c["B"] * (c["S"] * c["pos0"] + c["S"] * (c["S"] + 1) // 2)
    return dict(bytes=cached * keys + 4 * M * qd, flops=4 * qd * pairs)


# ---- 4 bits in plain operations ----------------------------------------------------------------------------------------------------

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)              # what the lower three bits of a code stand for; the fourth is the sign


def _parts(pages, c):
    """Views of pages [..., bytes]: codes [..., TK, Dh / 2] and scales [..., TK, Dh / 16]."""
    n = c["TK"] * c["Dh"] // 2
    return pages[..., :n].unflatten(-1, (c["TK"], c["Dh"] // 2)), pages[..., n:].view(torch.float8_e4m3fn).unflatten(-1, (c["TK"], c["Dh"] // 16))


def _quantise(x, exp):
    """bf16 values [..., Dh] as codes [..., Dh / 2] and scales [..., Dh / 16]: the scale is the group's largest magnitude over 6, both
    roundings go to the nearest, ties to the even code."""
    g = (x.float() * 2.0 ** -exp).unflatten(-1, (-1, 16))
    scale = (g.abs().amax(-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = scale.float().unsqueeze(-1)
    q = torch.where(s > 0, g / s, torch.zeros_like(g))
    a = q.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0) + 8 * torch.signbit(q)
    code = code.flatten(-2).unflatten(-1, (-1, 2))
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scale


def _values(codes, scales, exp):
    """What codes and scales stand for, in 32 bits."""
    nibbles = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()
    level = torch.tensor(LEVELS, device=codes.device).index_select(0, (nibbles & 7).flatten()).view(nibbles.shape)
    value = torch.where(nibbles >= 8, -level, level)
    return (value.unflatten(-1, (-1, 16)) * scales.float().unsqueeze(-1) * 2.0 ** exp).flatten(-2)


def _cache(tiles, c, n, exp):
    """The first n positions of tiles [n_tiles, B, Hkv, bytes] in 32 bits, [B, Hkv, n, Dh]."""
    codes, scales = _parts(tiles, c)
    return _values(codes, scales, exp).movedim(0, 2).flatten(2, 3)[:, :, :n]


# ---- the operators in plain form ---------------------------------------------------------------------------------------------------

def _append(st):
    c = st["case"]
    B, S, half = c["B"], c["S"], c["Dh"] // 2
    first = st["pos"].long() if c["ragged"] else torch.full((B,), c["pos0"], device="cuda")
    at = first[:, None] + torch.arange(S, device="cuda")                                 # [B, S]
    live = (first >= 0)[:, None, None, None]
    cos, sin = (t.double()[at.clamp(min=0)][:, :, None] for t in (st["cos"], st["sin"]))

    def rotated(x, H):                                         # in 64 bits: a value next to the border of two roundings
        x = x.view(B, S, H, c["Dh"]).double()
        lo, hi = x[..., :half], x[..., half:]
        return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1).float().bfloat16()

    st["qb"].copy_(torch.where(live, rotated(st["q"], c["Hq"]), st["qb"].view(B, S, c["Hq"], -1)).flatten(1).view(B * S, -1))
    keep = (first >= 0).nonzero().flatten()
    rows = at[keep]
    for x, tiles, exp, out in ((rotated(st["k"], c["Hkv"]), st["kt"], c["k_exp"], st["kb"]),
                               (st["v"].view(B, S, c["Hkv"], -1).bfloat16(), st["vt"], c["v_exp"], st["vb"])):
        codes, scales = _quantise(x[keep], exp)
        tile_codes, tile_scales = _parts(tiles, c)
        tile_codes[rows // c["TK"], keep[:, None], :, rows % c["TK"]] = codes
        tile_scales.view(torch.uint8)[rows // c["TK"], keep[:, None], :, rows % c["TK"]] = scales.view(torch.uint8)
        out[keep] = _values(codes, scales, exp).bfloat16().movedim(1, 2)
    return dict(q=st["qb"], k=st["kb"], v=st["vb"])


def _attn(st):
    c = st["case"]
    B, S, Hkv, G, n = c["B"], c["S"], c["Hkv"], c["Hq"] // c["Hkv"], c["pos0"] + c["S"]
    first = st["pos"].long() if c["ragged"] else torch.full((B,), c["pos0"], device="cuda")
    q = st["qb"].view(B, S, Hkv, G, c["Dh"]).float().permute(0, 2, 1, 3, 4).flatten(2, 3)
    scores = q @ _cache(st["kt"], c, n, c["k_exp"]).transpose(-1, -2) / math.sqrt(c["Dh"])               # [B, Hkv, S * G, n]
    last = first[:, None] + torch.arange(S, device="cuda")
    seen = (torch.arange(n, device="cuda") <= last[:, :, None]) & (first >= 0)[:, None, None]
    seen = seen.repeat_interleave(G, 1)[:, None]
    scores = torch.where(seen, scores, torch.full_like(scores, -math.inf))
    p = torch.where(seen, torch.exp(scores - scores.amax(-1, keepdim=True)), torch.zeros_like(scores))
    total = p.sum(-1, keepdim=True)
    o = p @ _cache(st["vt"], c, n, c["v_exp"]) / torch.where(total > 0, total, torch.ones_like(total))
    st["ob"].copy_(o.unflatten(2, (S, G)).permute(0, 2, 1, 3, 4).flatten(2).view(B * S, -1).bfloat16())
    return st["ob"]


def _move(st):
    c = st["case"]
    src, dst = st["index"]
    end = (c["len"] - 1) % c["TK"] + 1                           # positions in use of the last tile
    for tiles in (st["kt"], st["vt"]):
        if c["form"] == "bf16":
            parts = [tiles]
        else:
            parts = [t.view(torch.uint8) for t in _parts(tiles, c)]
        for rows in parts:                                       # [n_tiles, B, Hkv, TK, elements of a row]
            for some in (rows[:-1], rows[-1:, :, :, :end]):
                if c["kind"] == "free":
                    some[:, dst] = 0
                else:
                    some[:, dst] = some[:, src]
    return dict(k=st["kt"], v=st["vt"])


def _sample(st):
    logits, u = st["logits"], st["u"].double()[:, None]
    B, V = logits.shape
    wide = lambda name, off: st[name][:, None] if name in st else torch.full((B, 1), off, device="cuda")       # noqa: E731
    t, k, p, least = wide("temperature", 1.0).double(), wide("top_k", 0), wide("top_p", 1.0).double(), wide("min_p", 0.0).double()
    x, order = torch.sort(logits, dim=1, descending=True, stable=True)
    greedy = t <= 0
    w = torch.exp((x.double() - x[:, :1].double()) / torch.where(greedy, torch.ones_like(t), t))
    rank = torch.arange(V, device="cuda")
    w = torch.where((k <= 0) | (rank < k), w, torch.zeros_like(w))
    sums = torch.cumsum(w, 1)
    keep = ((p >= 1) | (sums - w < p * sums[:, -1:])) & (w >= least) & (w > 0) & ~greedy | (rank == 0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, torch.zeros_like(w)))
    sums = torch.cumsum(w, 1)
    st["token"].copy_((sums <= u * sums[:, -1:]).sum(1).clamp(max=V - 1))
    return st["token"]


# ---- the same by the framework ------------------------------------------------------------------------------------------------------

def _own(st):
    from paper_2609_06172_b200 import binding as tb
    c, stream = st["case"], torch.cuda.current_stream()
    if c["op"] == "sample":
        tb.k_sample(st["logits"], st["u"], st["token"], c["B"], c["V"], st.get("temperature"), st.get("top_k"), st.get("top_p"), st.get("min_p"), stream)
        return st["token"]
    if "cfg" not in st:                                          # what a user's program keeps: the model's sizes and a workspace
        n = c["TK"] * len(st["k_tiles"])
        st["cfg"] = tb.ModelCfg(L=1, d=c["Hq"] * c["Dh"], Hq=c["Hq"], Hkv=c["Hkv"], Dh=c["Dh"], F=1, V=1, E=0, topk=0, B=c["B"], max_len=n, TK=c["TK"],
                                rope_base=10000.0, eps=1e-5)
        if c["op"] == "attn":
            st["scratch"] = torch.empty(tb.k_attn_q4_scratch_bytes(st["cfg"], c["S"]), dtype=torch.uint8, device="cuda")
    cfg = st["cfg"]
    if c["op"] == "move":
        tb.k_kv_move(st["k_tiles"], st["v_tiles"], st["src"], st["dst"], cfg, tb.KV_Q4 if c["form"] == "q4" else tb.KV_BF16, c["B"], c["len"], stream)
        return dict(k=st["kt"], v=st["vt"])
    if c["op"] == "append":
        tb.k_rope_kv_q4(st["q"], st["k"], st["v"], st["qb"], st["k_tiles"], st["v_tiles"], st["cos"], st["sin"], cfg, c["B"], c["S"], c["pos0"],
                        c["k_exp"], c["v_exp"], st["pos"], stream)
        tb.k_kv_unpack_q4(st["k_tiles"], st["v_tiles"], st["kb"], st["vb"], cfg, c["B"], c["S"], c["pos0"], c["k_exp"], c["v_exp"], st["pos"], stream)
        return dict(q=st["qb"], k=st["kb"], v=st["vb"])
    tb.k_attn_q4(st["qb"], st["k_tiles"], st["v_tiles"], st["ob"], cfg, c["B"], c["S"], c["pos0"], c["k_exp"], c["v_exp"], st["pos"], st["scratch"], stream)
    return st["ob"]


def run(state):
    if own:
        return _own(state)
    return {"append": _append, "attn": _attn, "move": _move, "sample": _sample}[state["case"]["op"]](state)


# ---- inputs --------------------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (_prepare_sample if case["op"] == "sample" else _prepare_cache)(case, gen)


def _prepare_sample(c, gen):
    """Logits of a trained model: most of the vocabulary far below a few candidates, more of them in some rows than in others."""
    B, V = c["B"], c["V"]
    uniform = lambda: torch.rand(B, device="cuda", generator=gen)                                              # noqa: E731
    spread = 1.5 + 2.0 * uniform()[:, None]
    st = dict(case=c, logits=torch.randn(B, V, device="cuda", generator=gen) * spread, u=uniform(), token=torch.zeros(B, dtype=torch.int32, device="cuda"))
    if c["filters"] != "none":
        st["temperature"] = 0.5 + uniform()
    if c["filters"] in ("top_k", "all", "mixed"):
        st["top_k"] = (1 + 99 * uniform()).int()
    if c["filters"] in ("top_p", "all", "mixed"):
        st["top_p"] = 0.5 + 0.49 * uniform()
    if c["filters"] in ("min_p", "all", "mixed"):
        st["min_p"] = 0.1 * uniform()
    if c["filters"] == "mixed":                                  # users who left one or another setting alone
        at = torch.arange(B, device="cuda")
        st["temperature"][at % 8 == 5] = 0.0
        st["top_k"][at % 2 == 0] = 0
        st["top_p"][at % 3 == 0] = 1.0
        st["min_p"][at % 4 < 3] = 0.0
    return st


def _prepare_cache(c, gen):
    B, Hkv, Dh, TK = c["B"], c["Hkv"], c["Dh"], c["TK"]
    n = c["len"] if c["op"] == "move" else c["pos0"] + c["S"]
    n_tiles = (n + TK - 1) // TK

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    def tiles(std, exp):
        if c.get("form") == "bf16":
            return normal(n_tiles, B, Hkv, TK, Dh, std=std, dtype=torch.bfloat16)
        out = torch.zeros(n_tiles, B, Hkv, TK * _row_bytes(c), dtype=torch.uint8, device="cuda")
        codes, scales = _parts(out, c)
        for j in range(n_tiles):
            channel = std * (0.5 + torch.rand(Hkv, 1, Dh, device="cuda", generator=gen))       # some dimensions of a head are larger than others
            x = (normal(B, Hkv, TK, Dh) * channel).bfloat16()
            a, b = _quantise(x, exp)
            codes[j].copy_(a)
            scales.view(torch.uint8)[j].copy_(b.view(torch.uint8))
        return out

    std_k, std_v = 1.5 * 2.0 ** c.get("k_exp", 0), 1.5 * 2.0 ** c.get("v_exp", 0)
    st = dict(case=c, kt=tiles(std_k, c.get("k_exp", 0)), vt=tiles(std_v, c.get("v_exp", 0)))
    st["k_tiles"], st["v_tiles"] = list(st["kt"]), list(st["vt"])
    if c["op"] == "move":
        pairs = _pairs(c)
        st["src"], st["dst"] = [a for a, _ in pairs], [b for _, b in pairs]
        st["index"] = torch.tensor(st["src"], device="cuda"), torch.tensor(st["dst"], device="cuda")
        return st
    st["pos"] = torch.from_numpy(_positions(c)).cuda() if c["ragged"] else None
    M, qd, kd = B * c["S"], c["Hq"] * Dh, Hkv * Dh
    if c["op"] == "attn":
        st["qb"] = normal(M, qd, std=1.5 / 2.0 ** c["k_exp"], dtype=torch.bfloat16)
        st["ob"] = torch.zeros(M, qd, dtype=torch.bfloat16, device="cuda")
        return st
    angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, Dh, 2, device="cuda", dtype=torch.float64) / Dh)
    st |= dict(q=normal(M, qd), k=normal(M, kd, std=std_k), v=normal(M, kd, std=std_v), cos=angle.cos().float(), sin=angle.sin().float(),
               qb=torch.zeros(M, qd, dtype=torch.bfloat16, device="cuda"))
    st["kb"], st["vb"] = torch.zeros(2, B, Hkv, c["S"], Dh, dtype=torch.bfloat16, device="cuda")
    return st


# ---- the operators from their definitions, in 64 bits ------------------------------------------------------------------------------

def _e4m3(code):
    """The number that the lower seven bits of an e4m3 code stand for."""
    e, m = code >> 3, code & 7
    return math.nan if code == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)


def _decoded(page, c, exp):
    """Pages [..., bytes] in 64 bits, [..., TK, Dh], by a table of what every byte holds."""
    two = torch.tensor([[s * LEVELS[v & 7] for v in (b & 15, b >> 4) for s in ((-1.0) ** (v >> 3),)] for b in range(256)], dtype=torch.float64, device="cuda")
    one = torch.tensor([(-1.0) ** (b >> 7) * _e4m3(b & 127) for b in range(256)], dtype=torch.float64, device="cuda")
    cut = c["TK"] * c["Dh"] // 2
    x = two[page[..., :cut].long()].view(*page.shape[:-1], c["TK"], c["Dh"])
    s = one[page[..., cut:].long()].view(*page.shape[:-1], c["TK"], c["Dh"] // 16)
    return x * s.repeat_interleave(16, -1) * 2.0 ** exp


def _nearest(x, levels):
    """Index of the nearest of ascending levels, the even one of two that are equally near; levels are all that there are."""
    levels = torch.tensor(levels, dtype=torch.float64, device=x.device)
    above = torch.searchsorted(levels, x).clamp(1, len(levels) - 1)
    far, near = (levels[above] - x), (x - levels[above - 1])
    return torch.where((far < near) | ((far == near) & (above % 2 == 0)), above, above - 1)


def exact(case, seed):
    st = prepare(case, seed)
    c = case
    if c["op"] == "sample":
        return _exact_sample(st)
    if c["op"] == "move":
        out = {name: st[t].clone() for name, t in (("k", "kt"), ("v", "vt"))}
        wide = c["Dh"] if c["form"] == "bf16" else c["Dh"] // 2
        for name, t in (("k", "kt"), ("v", "vt")):
            for a, b in _pairs(c):
                for j in range(len(st[t])):
                    used = min(c["TK"], c["len"] - j * c["TK"])
                    old, new = st[t][j, max(a, 0)].flatten(1), out[name][j, b].flatten(1)
                    spans = [(0, used * wide)] + ([(c["TK"] * wide, c["TK"] * wide + used * c["Dh"] // 16)] if c["form"] == "q4" else [])
                    for lo, hi in spans:
                        new[:, lo:hi] = old[:, lo:hi] if a >= 0 else 0
        return out
    first = _positions(c) if c["ragged"] else np.full(c["B"], c["pos0"])
    return (_exact_append if c["op"] == "append" else _exact_attn)(st, c, first)


def _exact_append(st, c, first):
    B, S, Dh = c["B"], c["S"], c["Dh"]
    shape = {"q": c["Hq"], "k": c["Hkv"], "v": c["Hkv"]}
    x = {name: st[name].view(B, S, H, Dh).double() for name, H in shape.items()}
    scales = [_e4m3(i) for i in range(127)]
    for b in range(B):
        if first[b] < 0:
            x["q"][b], x["k"][b], x["v"][b] = 0, 0, 0
            continue
        at = slice(int(first[b]), int(first[b]) + S)
        turn = torch.complex(st["cos"][at].double(), st["sin"][at].double())[:, None]
        for name in ("q", "k"):
            y = torch.complex(x[name][b, ..., :Dh // 2], x[name][b, ..., Dh // 2:]) * turn
            x[name][b] = torch.cat((y.real, y.imag), -1)
    out = {"q": x["q"].float().bfloat16().double().view(B * S, -1)}
    for name, exp in (("k", c["k_exp"]), ("v", c["v_exp"])):
        g = x[name].float().bfloat16().double().view(B, S, c["Hkv"], Dh // 16, 16) / 2.0 ** exp
        s = torch.tensor(scales, dtype=torch.float64, device="cuda")[_nearest(g.abs().amax(-1) / 6, scales)].unsqueeze(-1)
        level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")[_nearest((g.abs() / s).nan_to_num(0.0), list(LEVELS))]
        out[name] = (g.sign() * level * s * 2.0 ** exp).flatten(-2).transpose(1, 2)
    return out


def _exact_attn(st, c, first):
    B, S, G, Dh = c["B"], c["S"], c["Hq"] // c["Hkv"], c["Dh"]
    out = torch.zeros(B, S, c["Hkv"], G, Dh, dtype=torch.float64, device="cuda")
    q = st["qb"].double().view(B, S, c["Hkv"], G, Dh)
    for b in range(B):
        if first[b] < 0:
            continue
        n = int(first[b]) + S
        k, v = (_decoded(st[t][:, b], c, e).transpose(0, 1).flatten(1, 2)[:, :n] for t, e in (("kt", c["k_exp"]), ("vt", c["v_exp"])))
        s = torch.einsum("thgd,hkd->htgk", q[b], k) * Dh ** -0.5
        s += torch.full((S, n), -math.inf, dtype=torch.float64, device="cuda").triu(n - S + 1)[:, None]
        out[b] = torch.einsum("htgk,hkd->thgd", torch.softmax(s, -1), v)
    return out.view(B * S, -1)


def _exact_sample(st):
    x, token = st["logits"].double().cpu().numpy(), np.zeros(len(st["u"]), dtype=np.int32)
    u = st["u"].double().cpu().numpy()
    given = {name: st[name].double().cpu().numpy() for name in ("temperature", "top_k", "top_p", "min_p") if name in st}
    for b in range(len(x)):
        t, k, p, least = (float(given[name][b]) if name in given else off for name, off in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)))
        if t <= 0:
            token[b] = np.argmax(x[b])
            continue
        order = np.lexsort((np.arange(x.shape[1]), -x[b]))
        order = order[:int(k)] if k > 0 else order
        w = np.exp((x[b, order] - x[b, order[0]]) / t)
        if p < 1:
            before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
            order, w = order[before < p * w.sum()], w[before < p * w.sum()]
        order, w = order[w >= least], w[w >= least]
        by_index = np.argsort(order)
        sums = np.cumsum(w[by_index])
        token[b] = order[by_index[np.searchsorted(sums, u[b] * sums[-1], side="right")]]
    return torch.from_numpy(token).cuda()
