"""A server over a KV cache in pages, whose users' requests differ in length and whose draft model proposes tokens: its operators as cases that
can be timed, each in a plain form and as a call of the framework.

  pages    pages taken and given back, and the places of a step's tokens, from the lengths of the requests
  append   a step's rows rotated, their keys and values put into the pages
  attn     attention of a ragged batch over the pages - single tokens, drafted tokens, prompts - over everything before, or a window and the first tokens
  verify   drafted tokens accepted or replaced by the target's and the draft's distributions from given random numbers

A page holds TK positions of one sequence and all KV heads, [Hkv, TK, Dh]; the pages of a layer are one array of keys and one of values.  A sequence's row of the
table lists its pages, position p being row p % TK of page table[b][p / TK].  The rows of a step lie one sequence behind the other: those of
sequence b are start[b] ... start[b + 1] - 1, at its positions up to end[b] - 1.

Head counts, dimensions and vocabularies are those of the repository's configurations or generic ones.
"""
import math

import torch

own = False

SMALL = dict(Hq=32, Hkv=8, Dh=64)              # heads of a 1B decoder
MEDIUM = dict(Hq=32, Hkv=8, Dh=128)            # heads of an 8B decoder
LARGE = dict(Hq=64, Hkv=8, Dh=128)             # heads of a 70B decoder


def listed():
    return [
        # a step of a busy server: everyone has a token and up to four drafted ones, some have left, some come with prompts; then the step is given up
        dict(name="pages_step_b61", op="pages", B=61, TK=16, max_len=4096, add=5, prompt=300, tokens=2048),
        # the prompts of many users at once, and users far into long documents beside them
        dict(name="pages_prompts_b512", op="pages", B=512, TK=16, max_len=32768, add=1, prompt=700, tokens=65536),
        # the rows of a step of 61 users with drafted tokens
        dict(MEDIUM, name="append_step_b61", op="append", B=61, S=5, ctx=2500, TK=64, kind="few"),
        # the prompts of nine users on a large model
        dict(LARGE, name="append_prompts_b9", op="append", B=9, S=1500, ctx=0, TK=16, kind="prompts"),
        # one user, one token, a short cache: nothing but latency
        dict(SMALL, name="attn_decode_b1", op="attn", B=1, S=1, ctx=700, TK=16, kind="few", window=0, sinks=0),
        # a busy server's step: users at lengths of their own
        dict(MEDIUM, name="attn_decode_b61", op="attn", B=61, S=1, ctx=2500, TK=64, kind="few", window=0, sinks=0),
        # 24 users far into long documents
        dict(LARGE, name="attn_decode_long_b24", op="attn", B=24, S=1, ctx=12000, TK=32, kind="few", window=0, sinks=0),
        # long chats of a model with a window and four first tokens that stay, with drafted tokens
        dict(MEDIUM, name="attn_window_drafts_b32", op="attn", B=32, S=5, ctx=14000, TK=16, kind="few", window=1024, sinks=4),
        # a chunk of prompt beside users who want their next token
        dict(MEDIUM, name="attn_mixed_b12", op="attn", B=12, S=509, ctx=1900, TK=64, kind="mixed", window=0, sinks=0),
        # prompts longer than the window, on a large model
        dict(LARGE, name="attn_window_prompts_b3", op="attn", B=3, S=2500, ctx=0, TK=128, kind="prompts", window=1000, sinks=4),
        # one user's four drafted tokens
        dict(name="verify_b1", op="verify", B=1, D=4, V=32000, draft="model", settings="one"),
        # a server's step: users with temperatures of their own over a large vocabulary
        dict(name="verify_b32", op="verify", B=32, D=4, V=128256, draft="model", settings="mixed"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """A case of the same ranges: one to 512 sequences, caches of one to 16000 positions, steps of one to 2500 rows a sequence, vocabularies of some thousands to 128256."""
    op = rng.choice(["pages", "append", "attn", "attn", "attn", "attn", "verify", "verify"])
    if op == "pages":
        B, TK = _log_int(rng, 1, 512), rng.choice([16, 32, 48, 64, 128])
        prompt = _log_int(rng, 10, 700)
        max_len = rng.choice([2048, 8192, 32768])
        return dict(op=op, B=B, TK=TK, max_len=max_len, add=rng.choice([1, 1, 5, 9]), prompt=prompt, tokens=min(65536, 64 + 9 * B + prompt * B // rng.choice([1, 4])))
    if op == "verify":
        V, D = _log_int(rng, 4001, 128256), rng.choice([1, 2, 4, 7])
        return dict(op=op, B=_log_int(rng, 1, min(64, 36_000_000 // (V * (2 * D + 1)))), D=D, V=V, draft=rng.choice(["model", "model", "none"]), settings=rng.choice(["one", "mixed", "greedy"]))
    Dh, Hkv, group = rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 5, 8])
    heads = dict(Hq=Hkv * group, Hkv=Hkv, Dh=Dh)
    kind, TK = rng.choice(["few", "few", "few", "mixed", "prompts"]), rng.choice([16, 32, 64, 128])
    if kind == "few":
        B, S = _log_int(rng, 1, 96), rng.choice([1, 1, 1, 2, 5, 9])
        ctx = _log_int(rng, 1, min(16000, 250_000_000 // (B * Hkv * Dh)))
    elif kind == "mixed":
        B, S = _log_int(rng, 2, 12), _log_int(rng, 20, 509)
        ctx = _log_int(rng, 100, 1900)
    else:
        B = _log_int(rng, 1, 9)
        S, ctx = _log_int(rng, 30, 6000 // (B + 1)), rng.choice([0, 0, _log_int(rng, 30, 1000)])
    case = dict(heads, op=op, B=B, S=S, ctx=ctx, TK=TK, kind=kind)
    if op == "attn":
        window = rng.choice([0, 0, _log_int(rng, 1, 2000)])
        case |= dict(window=window, sinks=rng.choice([0, 1, 4, 20]) if window else 0)
    return case


# ---- what a case says besides its sizes -----------------------------------------------------------------------------------------

def _spread(i, lo, hi):
    """A number of [lo, hi] for place i of a batch, evenly spread."""
    return lo + int((i * 0.6180339887 % 1.0) * (hi - lo + 1))


def _rows(case):
    """Of each sequence of an append or attention: its new rows, and its length behind them."""
    B, S, ctx, out = case["B"], case["S"], case["ctx"], []
    for b in range(B):
        if b == 0:
            n, before = S, ctx
        elif case["kind"] == "few":
            n, before = (S if b % 3 else 1), _spread(b, ctx // 8, ctx)
            n = 0 if b % 13 == 7 else n                          # a place of the batch without a request
        elif case["kind"] == "mixed":
            n, before = (S if b % 6 == 0 else 1), _spread(b, 0, ctx)
        else:
            n, before = _spread(b, S // 4 + 1, S), _spread(b, 0, ctx)
        out.append((n, before + n))
    return out


def _sizes(case):
    rows = _rows(case)
    T, kv_max, q_max = sum(n for n, _ in rows), max(e for _, e in rows), max(n for n, _ in rows)
    P = case["TK"]
    return rows, T, kv_max, q_max, sum(-(-e // P) for _, e in rows) + 3          # (pages: a few belong to nobody)


def _lengths(case):
    """Of each sequence of a page plan: positions that stay, new ones, and positions that its pages are for now."""
    out = []
    for b in range(case["B"]):
        have = _spread(b, 1, case["max_len"] // 4)
        if b % 8 == 3:
            out.append((0, 0, have))                             # has left
        elif b % 8 == 6:
            out.append((0, min(case["prompt"], _spread(b, 1, case["prompt"])), 0))       # comes with a prompt
        elif b % 8 == 1:
            out.append((have - min(have, 3), 1, have))           # takes back what was not accepted
        else:
            out.append((have, 1 + b % case["add"], have))
    return out


def _seen(case, pos):
    """Keys that the query at a position sees."""
    return pos + 1 if not case["window"] or pos < case["window"] + case["sinks"] else case["window"] + case["sinks"]


def work(case):
    c = case
    if c["op"] == "verify":
        rows = c["B"] * (2 * c["D"] + (1 if c["draft"] == "model" else -c["D"] + 1))
        return dict(bytes=4 * c["V"] * rows + 16 * c["B"] * (c["D"] + 1), flops=2 * c["V"] * rows)
    if c["op"] == "pages":
        P, lens = c["TK"], _lengths(c)
        moved = sum(abs(-(-(n + a) // P) - -(-h // P)) + -(-a // P) for n, a, h in lens)
        return dict(bytes=16 * c["B"] + 16 * moved + 8 * c["tokens"], flops=0)
    rows, T, _, _, _ = _sizes(c)
    qd, kd = c["Hq"] * c["Dh"], c["Hkv"] * c["Dh"]
    if c["op"] == "append":
        return dict(bytes=T * (6 * qd + 12 * kd + 8) + 4 * c["Dh"] * len({p for n, e in rows for p in range(e - n, e)}), flops=6 * T * (qd + kd))
    pairs = keys = 0
    for n, e in rows:
        if n:
            pairs += sum(_seen(c, p) for p in range(e - n, e))
            first = e - n - c["window"] + 1                      # the first position of the window of the first query
            keys += e if not c["window"] or first <= c["sinks"] else e - first + c["sinks"]
    return dict(bytes=4 * kd * keys + 4 * T * qd, flops=4 * qd * pairs)


# ---- the operators in plain form ---------------------------------------------------------------------------------------------------

def _plan(st, length, add):
    """One call: pages given back go to the top of the stack of free ones, pages needed come from there; then the places of the new positions."""
    c, table, held, free, n_free = st["case"], st["table"], st["held"], st["free"], st["n_free"]
    B, P, T, n_pages, W = c["B"], c["TK"], c["tokens"], len(free), table.shape[1]
    length, add, had = length.long(), add.long(), held.long()
    valid = (length >= 0) & (add >= 0) & (length + add <= c["max_len"])
    want = torch.where(valid, (length + add + P - 1) // P, had)
    column = torch.arange(W, device="cuda")[None]

    given = (column >= want[:, None]) & (column < had[:, None])
    top = n_free.long() + given.sum()
    order = given.flatten().cumsum(0).view(B, W) - 1
    stack = torch.cat((free, free.new_zeros(1)))                 # (the last entry takes what goes nowhere)
    stack.scatter_(0, torch.where(given, top - 1 - order, torch.full_like(order, n_pages)).flatten(), table.flatten())
    table.copy_(torch.where(given, torch.full_like(table, -1), table))

    need = (want - had).clamp(min=0)
    asked = torch.where(valid, add, torch.zeros_like(add))
    served = valid & ((need == 0) | (need.cumsum(0) <= top)) & ((add == 0) | (asked.cumsum(0) <= T))
    n, take = (torch.where(served, x, torch.zeros_like(x)) for x in (add, need))
    new = served[:, None] & (column >= had[:, None]) & (column < want[:, None])
    order = (take.cumsum(0) - take)[:, None] + column - had[:, None]
    table.copy_(torch.where(new, stack[(top - 1 - order).clamp(0, n_pages)], table))
    held.copy_(torch.where(served | (want < had), want, had))
    free.copy_(stack[:n_pages])
    n_free.copy_(top - take.sum())

    start = torch.cat((n.new_zeros(1), n.cumsum(0)))
    st["start"].copy_(start)
    st["end"].copy_(length + n)
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(start[1:], t, right=True).clamp(max=B - 1)
    pos = length[b] + t - start[b]
    slot = table[b, (pos // P).clamp(0, W - 1)].long() * P + pos % P
    st["pos"].copy_(torch.where(t < start[-1], pos, torch.full_like(pos, -1)))
    st["slot"].copy_(torch.where(t < start[-1], slot, torch.full_like(slot, -1)))


def _pages_outputs(st):
    return dict(table=st["table"], held=st["held"], free=st["free"], n_free=st["n_free"])


def _pages(st):
    _plan(st, st["length"], st["add"])
    step = {k: st[k].clone() for k in ("start", "end", "slot", "pos", "table")}
    _plan(st, st["length"], st["nothing"])
    return dict(step=step, after=_pages_outputs(st))


def _append(st):
    c = st["case"]
    half, live = c["Dh"] // 2, (st["slot"] >= 0).nonzero().flatten()
    at, slot = st["pos"][live].long(), st["slot"][live].long()
    cos, sin = st["cos"].double()[at][:, None], st["sin"].double()[at][:, None]

    def rotated(x, H):                                           # in 64 bits: a value next to the border of two roundings
        x = x[live].view(-1, H, c["Dh"]).double()
        lo, hi = x[..., :half], x[..., half:]
        return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1).bfloat16()

    st["qb"][live] = rotated(st["q"], c["Hq"]).flatten(1)
    st["k_pages"][slot // c["TK"], :, slot % c["TK"]] = rotated(st["k"], c["Hkv"])
    st["v_pages"][slot // c["TK"], :, slot % c["TK"]] = st["v"][live].view(-1, c["Hkv"], c["Dh"]).bfloat16()
    return dict(q=st["qb"], k=st["k_pages"], v=st["v_pages"])


def _attn(st):
    c = st["case"]
    B, Hkv, G, Dh, S, T = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["Dh"], st["q_max"], st["T"]
    start, end = st["start"].long(), st["end"].long()
    i = torch.arange(S, device="cuda")
    there = i < (start[1:] - start[:-1])[:, None]                                                        # [B, S]
    row = torch.where(there, start[:-1, None] + i, torch.full_like(start[:-1, None] + i, T))
    pos = end[:, None] - (start[1:] - start[:-1])[:, None] + i
    pages = st["table"][:, :-(-st["kv_max"] // c["TK"])].long().clamp(min=0)

    def cache(x):                                                                                        # [B, Hkv, n, Dh]
        return x[pages].float().movedim(2, 1).flatten(2, 3)

    q = st["qb"][row.clamp(max=T - 1)].view(B, S, Hkv, G, Dh).float().permute(0, 2, 1, 3, 4).flatten(2, 3)
    scores = q @ cache(st["k_pages"]).transpose(-1, -2) / math.sqrt(Dh)                                  # [B, Hkv, S * G, n]
    j = torch.arange(scores.shape[-1], device="cuda")
    seen = (j <= pos[:, :, None]) & there[:, :, None]
    if c["window"]:
        seen &= (j > pos[:, :, None] - c["window"]) | (j < c["sinks"])
    seen = seen.repeat_interleave(G, 1)[:, None]
    scores = torch.where(seen, scores, torch.full((), -math.inf, device="cuda"))
    p = torch.where(seen, torch.exp(scores - scores.amax(-1, keepdim=True)), torch.zeros((), device="cuda"))
    total = p.sum(-1, keepdim=True)
    o = p @ cache(st["v_pages"]) / torch.where(total > 0, total, torch.ones_like(total))
    out = torch.cat((st["ob"], st["ob"][:1]))                                                            # (the last row takes what no row is for)
    out[row.flatten()] = o.unflatten(2, (S, G)).permute(0, 2, 1, 3, 4).reshape(B * S, -1).bfloat16()
    st["ob"].copy_(out[:-1])
    return st["ob"]


def _verify(st):
    x, y, tokens, start = st["logits"], st["draft_logits"], st["tokens"].long(), st["start"].long()
    T, V = x.shape
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(start[1:], t, right=True)
    judged = t + 1 < start[1:][b]                                # the row has a drafted token behind it
    token = tokens[(t + 1).clamp(max=T - 1)]
    temperature = st["temperature"].double() if st["temperature"] is not None else torch.ones(len(start) - 1, dtype=torch.float64, device="cuda")
    greedy, scale = temperature <= 0, torch.where(temperature > 0, temperature, torch.ones_like(temperature))

    def probabilities(z):
        w = torch.exp((z.double() - z.amax(1, keepdim=True).double()) / scale[b][:, None])
        return w / w.sum(1, keepdim=True)

    p, best = probabilities(x), x.argmax(1)
    q = probabilities(y) if y is not None else torch.zeros_like(p).scatter_(1, token[:, None], 1.0)
    of = lambda z: z.gather(1, token[:, None])[:, 0]             # noqa: E731
    accepted = torch.where(greedy[b], token == best, st["u"].double() * of(q) < of(p))
    stop = torch.where(judged & accepted, torch.full_like(t, T), t)
    row = torch.full_like(start[1:], T).scatter_reduce_(0, b, stop, "amin")          # the row that each sequence's last token comes from
    rest = torch.where(judged[row][:, None], (p[row] - q[row]).clamp(min=0), p[row])
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, p[row])
    sums = rest.cumsum(1)
    drawn = (sums <= st["u_draw"].double()[:, None] * sums[:, -1:]).sum(1).clamp(max=V - 1)
    last = torch.where(greedy, best[row], drawn)
    st["out"].copy_(torch.where(t < row[b], token, torch.where(t == row[b], last[b], torch.full_like(t, -1))))
    st["n_out"].copy_(row - start[:-1] + 1)
    return dict(out=st["out"], n_out=st["n_out"])


# ---- the same by the framework ------------------------------------------------------------------------------------------------------

def _own(st):
    from paper_2609_06172_b200 import binding as tb
    c, stream = st["case"], torch.cuda.current_stream()
    if c["op"] == "verify":
        T, V = st["logits"].shape
        if "scratch" not in st:                                  # what a user's program keeps: a workspace, and the model's sizes below
            st["scratch"] = torch.empty(tb.k_verify_scratch_bytes(T, V), dtype=torch.uint8, device="cuda")
        tb.k_verify(st["logits"], st["draft_logits"], st["tokens"], st["start"], st["u"], st["u_draw"], st["out"], st["n_out"], c["B"], T, V, st["temperature"],
                    st["scratch"], stream)
        return dict(out=st["out"], n_out=st["n_out"])
    if "cfg" not in st:
        heads = {k: c.get(k, 1) for k in ("Hq", "Hkv")} | dict(Dh=c.get("Dh", 64))
        st["cfg"] = tb.ModelCfg(L=1, d=heads["Hq"] * heads["Dh"], **heads, F=1, V=1, E=0, topk=0, B=c["B"], max_len=c.get("max_len") or st["kv_max"], TK=c["TK"],
                                rope_base=10000.0, eps=1e-5)
        if c["op"] == "attn":
            st["scratch"] = torch.empty(tb.k_attn_paged_scratch_bytes(st["cfg"], c["B"], st["T"], st["q_max"], st["kv_max"]), dtype=torch.uint8, device="cuda")
    cfg = st["cfg"]
    if c["op"] == "pages":
        def plan(add):
            tb.k_page_plan(st["length"], add, st["table"], st["held"], st["free"], st["n_free"], st["start"], st["end"], st["slot"], st["pos"], cfg, c["B"], len(st["free"]),
                           c["tokens"], stream)
        plan(st["add"])
        step = {k: st[k].clone() for k in ("start", "end", "slot", "pos", "table")}
        plan(st["nothing"])
        return dict(step=step, after=_pages_outputs(st))
    if c["op"] == "append":
        tb.k_rope_kv_paged(st["q"], st["k"], st["v"], st["qb"], st["k_pages"], st["v_pages"], st["cos"], st["sin"], st["slot"], st["pos"], cfg, st["T"], st["n_pages"], stream)
        return dict(q=st["qb"], k=st["k_pages"], v=st["v_pages"])
    tb.k_attn_paged(st["qb"], st["k_pages"], st["v_pages"], st["ob"], st["table"], st["start"], st["end"], cfg, c["B"], st["T"], st["q_max"], st["kv_max"], st["n_pages"],
                    c["window"], c["sinks"], st["scratch"], stream)
    return st["ob"]


def run(state):
    if own:
        return _own(state)
    return {"pages": _pages, "append": _append, "attn": _attn, "verify": _verify}[state["case"]["op"]](state)


# ---- inputs --------------------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"pages": _prepare_pages, "verify": _prepare_verify}.get(case["op"], _prepare_cache)(case, gen)


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pages_of(lengths, P, W, n_pages, gen):
    """Pages at random for sequences of these lengths, [B, W], and the others."""
    order = torch.randperm(n_pages, device="cuda", generator=gen).int()
    counts = _int([-(-n // P) for n in lengths])
    column = torch.arange(W, device="cuda")[None]
    at = (counts.cumsum(0) - counts)[:, None] + column
    table = torch.where(column < counts[:, None], order[at.clamp(max=n_pages - 1)], torch.full_like(at, -1, dtype=torch.int32))
    return table, counts, order[int(counts.sum()):]


def _prepare_pages(c, gen):
    """A server with hardly more pages than its users have now: where few leave, the last of those that come have to wait."""
    B, P = c["B"], c["TK"]
    shift = [int(v) for v in torch.randint(0, 3, (B,), device="cuda", generator=gen).tolist()]            # lengths differ from seed to seed
    lens = [(max(0, n - s) if n else 0, a, max(n, h - s) if n else h) for (n, a, h), s in zip(_lengths(c), shift)]
    most = [(-(-(n + a) // P), -(-h // P)) for n, a, h in _lengths(c)]
    n_pages = sum(h for _, h in most) + max(0, sum(max(0, n - h) for n, h in most) * 7 // 8 - sum(max(0, h - n) for n, h in most)) + 1
    table, counts, rest = _pages_of([h for _, _, h in lens], P, -(-c["max_len"] // P), n_pages, gen)
    st = dict(case=c, length=_int([n for n, _, _ in lens]), add=_int([a for _, a, _ in lens]), nothing=_int([0] * B), table=table, held=counts,
              free=torch.cat((rest, rest.new_full((n_pages - len(rest),), -1))), n_free=_int([len(rest)]),
              start=_int([0] * (B + 1)), end=_int([0] * B), slot=_int([0] * c["tokens"]), pos=_int([0] * c["tokens"]))
    return st


def _prepare_verify(c, gen):
    """Logits of a trained model, a draft model near it, and the tokens that the draft drew from its own distribution."""
    B, D, V = c["B"], c["D"], c["V"]
    n = [D + 1 if b % 5 != 3 else 1 + b % (D + 1) for b in range(B)]                                     # some drafts are shorter
    T, start = sum(n), [sum(n[:b]) for b in range(B + 1)]
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), _int(n).long())
    uniform = lambda *shape: torch.rand(*shape, device="cuda", generator=gen)                            # noqa: E731
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)                            # noqa: E731
    spread = 1.5 + 2.0 * uniform(T)[:, None]
    logits = normal(T, V) * spread
    draft = logits + 0.5 * normal(T, V)
    temperature = None
    if c["settings"] != "one":
        temperature = 0.5 + uniform(B)
        temperature[(torch.arange(B, device="cuda") % 8 == 5) | (c["settings"] == "greedy")] = 0.0
    each = temperature[seq] if temperature is not None else torch.ones(T, device="cuda")
    noise = -torch.log(-torch.log(uniform(T, V).clamp(1e-12, 1 - 1e-7)))                                 # (the largest of logits plus this noise is a draw)
    drawn = (draft / each.clamp(min=1e-3)[:, None] + torch.where(each > 0, 1.0, 0.0)[:, None] * noise).argmax(1)
    tokens = torch.cat((torch.randint(0, V, (1,), device="cuda", generator=gen), drawn[:-1])).int()      # row r + 1 holds what was drawn behind row r
    return dict(case=c, logits=logits, draft_logits=draft if c["draft"] == "model" else None, tokens=tokens, start=_int(start), u=uniform(T), u_draw=uniform(B),
                temperature=temperature, out=_int([0] * T), n_out=_int([0] * B))


def _prepare_cache(c, gen):
    rows, T, kv_max, q_max, n_pages = _sizes(c)
    Hq, Hkv, Dh, P = c["Hq"], c["Hkv"], c["Dh"], c["TK"]

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    table, _, _ = _pages_of([e for _, e in rows], P, -(-kv_max // P), n_pages, gen)
    starts = [sum(n for n, _ in rows[:b]) for b in range(len(rows) + 1)]
    st = dict(case=c, T=T, kv_max=kv_max, q_max=q_max, n_pages=n_pages, table=table, start=_int(starts), end=_int([e for _, e in rows]),
              k_pages=normal(n_pages, Hkv, P, Dh, std=1.5, dtype=torch.bfloat16), v_pages=normal(n_pages, Hkv, P, Dh, std=1.5, dtype=torch.bfloat16))
    if c["op"] == "attn":
        st["qb"] = normal(T, Hq * Dh, std=1.5, dtype=torch.bfloat16)
        st["ob"] = torch.zeros(T, Hq * Dh, dtype=torch.bfloat16, device="cuda")
        return st
    spare = 1 + T // 16                                          # a step's buffers hold more rows than there are tokens
    pos = [p for n, e in rows for p in range(e - n, e)]
    seq = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), _int([n for n, _ in rows]).long())
    at = _int(pos).long()
    slot = table[seq, at // P] * P + (at % P).int()
    st["pos"], st["slot"] = _int(pos + [-1] * spare), torch.cat((slot, slot.new_full((spare,), -1)))
    angle = torch.arange(kv_max, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, Dh, 2, device="cuda", dtype=torch.float64) / Dh)
    T = st["T"] = T + spare
    st |= dict(q=normal(T, Hq * Dh), k=normal(T, Hkv * Dh, std=1.5), v=normal(T, Hkv * Dh, std=1.5), cos=angle.cos().float(), sin=angle.sin().float(),
               qb=torch.zeros(T, Hq * Dh, dtype=torch.bfloat16, device="cuda"))
    return st


# ---- the operators from their definitions, in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"pages": _exact_pages, "append": _exact_append, "attn": _exact_attn, "verify": _exact_verify}[case["op"]](st, case)


def _exact_pages(st, c):
    """Sequence by sequence, with lists."""
    length, add, table = st["length"].tolist(), st["add"].tolist(), [[p for p in row if p >= 0] for row in st["table"].tolist()]
    W, n_pages = st["table"].shape[1], len(st["free"])
    stack, behind = st["free"].tolist()[:int(st["n_free"])], st["free"].tolist()

    def plan(add):
        given = []
        for b, pages in enumerate(table):
            want = -(-(length[b] + add[b]) // c["TK"])
            given += pages[want:]
            del pages[want:]
        stack.extend(reversed(given))
        behind[:len(stack)] = stack
        left, room, start, slot, pos = len(stack), c["tokens"], [0], [], []
        for b, pages in enumerate(table):
            need = max(0, -(-(length[b] + add[b]) // c["TK"]) - len(pages))
            left, room = left - need, room - add[b]
            n = add[b] if (not need or left >= 0) and (not add[b] or room >= 0) else 0
            if n:
                pages.extend(stack.pop() for _ in range(need))
            pos += range(length[b], length[b] + n)
            slot += [pages[p // c["TK"]] * c["TK"] + p % c["TK"] for p in range(length[b], length[b] + n)]
            start.append(len(pos))
        rest = [-1] * (c["tokens"] - len(pos))
        return dict(start=_int(start), end=_int([n + e - s for n, s, e in zip(length, start, start[1:])]), slot=_int(slot + rest), pos=_int(pos + rest), table=tables())

    def tables():
        return _int([pages + [-1] * (W - len(pages)) for pages in table])

    step = plan(add)
    plan([0] * len(add))
    return dict(step=step, after=dict(table=tables(), held=_int([len(p) for p in table]), free=_int(behind), n_free=_int([len(stack)])))


def _exact_append(st, c):
    half, out = c["Dh"] // 2, dict(q=st["qb"].double(), k=st["k_pages"].double(), v=st["v_pages"].double())
    turn = torch.complex(st["cos"].double(), st["sin"].double())
    rows = [(t, s, p) for t, (s, p) in enumerate(zip(st["slot"].tolist(), st["pos"].tolist())) if s >= 0]
    t, s, p = (torch.tensor(v, device="cuda") for v in zip(*rows))
    for name, source, H in (("q", "q", c["Hq"]), ("k", "k", c["Hkv"])):
        x = st[source][t].double().view(-1, H, c["Dh"])
        y = torch.complex(x[..., :half], x[..., half:]) * turn[p][:, None]
        y = torch.cat((y.real, y.imag), -1)
        if name == "q":
            out["q"][t] = y.flatten(1)
        else:
            out["k"][s // c["TK"], :, s % c["TK"]] = y
    out["v"][s // c["TK"], :, s % c["TK"]] = st["v"][t].double().view(-1, c["Hkv"], c["Dh"])
    return out


def _exact_attn(st, c):
    G, Dh = c["Hq"] // c["Hkv"], c["Dh"]
    out = torch.zeros(st["T"], c["Hkv"], G, Dh, dtype=torch.float64, device="cuda")
    start, end = st["start"].tolist(), st["end"].tolist()
    for b in range(c["B"]):
        n, e = start[b + 1] - start[b], end[b]
        if not n:
            continue
        pages = st["table"][b, :-(-e // c["TK"])].long()
        k, v = (st[x][pages].double().transpose(0, 1).flatten(1, 2)[:, :e] for x in ("k_pages", "v_pages"))
        hidden = torch.ones(n, e, dtype=torch.bool, device="cuda").triu(e - n + 1)
        if c["window"]:
            far = torch.ones(n, e, dtype=torch.bool, device="cuda").tril(e - n - c["window"])
            far[:, :c["sinks"]] = False
            hidden |= far
        for i in range(0, n, 256):                               # (256 queries at a time: the scores of all would not fit)
            q = st["qb"][start[b] + i:min(start[b] + i + 256, start[b + 1])].double().view(-1, c["Hkv"], G, Dh)
            s = torch.einsum("thgd,hkd->htgk", q, k) * Dh ** -0.5
            s.masked_fill_(hidden[i:i + 256, None], -math.inf)
            out[start[b] + i:start[b] + i + len(q)] = torch.einsum("htgk,hkd->thgd", torch.softmax(s, -1), v)
    return out.flatten(1)


def _exact_verify(st, c):
    """Sequence by sequence, token by token."""
    start, tokens, u, u_draw = st["start"].tolist(), st["tokens"].tolist(), st["u"].double().tolist(), st["u_draw"].double().tolist()
    out, n_out = [], []
    for b in range(c["B"]):
        t = 1.0 if st["temperature"] is None else float(st["temperature"][b])
        answer = []
        for r in range(start[b], start[b + 1]):
            x, judged = st["logits"][r].double(), r + 1 < start[b + 1]
            best = int((x == x.max()).nonzero()[0])
            d = tokens[r + 1] if judged else -1
            if t <= 0:
                answer.append(best)
                if d != best:
                    break
                continue
            p = torch.softmax(x / t, 0)
            if judged:
                q = torch.softmax(st["draft_logits"][r].double() / t, 0) if st["draft_logits"] is not None else torch.nn.functional.one_hot(torch.tensor(d, device="cuda"), c["V"]).double()
                if u[r] * float(q[d]) < float(p[d]):
                    answer.append(d)
                    continue
                p = (p - q).clamp(min=0)
            sums = torch.cumsum(p, 0)
            answer.append(int(torch.searchsorted(sums, u_draw[b] * sums[-1], right=True)))
            break
        out += answer + [-1] * (start[b + 1] - start[b] - len(answer))
        n_out.append(len(answer))
    return dict(out=_int(out), n_out=_int(n_out))
