"""4-bit KV tiles on the GPU - append, read back, attention, moves - against plain 64-bit arithmetic (oracle/kv_q4.py), at the sizes and values where they can go
wrong, and a batch that answers with samples, as the operators would be used together."""
import numpy as np
import pytest

import seeded_inputs as si

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import kv_q4, sample  # noqa: E402
from oracle.forward import bf16_round  # noqa: E402
from paper_2609_06172_b200 import binding as tb  # noqa: E402

DEV = "cuda:0"
HALF_BF16, HALF_FP16 = 2.0 ** -8, 2.0 ** -11               # half a step, relative to the value


def config(Hq=8, Hkv=2, Dh=64, B=2, max_len=256, TK=32):
    return tb.ModelCfg(L=1, d=Hq * Dh, Hq=Hq, Hkv=Hkv, Dh=Dh, F=1, V=1, E=0, topk=0, B=B, max_len=max_len, TK=TK, rope_base=10000.0, eps=1e-5)


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV).bfloat16()


def f32(t):
    return t.float().cpu().numpy()


def random_tiles(rng, c, n_tiles, exp, std=1.0):
    """Tiles of quantised normal values, as host pages [n_tiles, B, Hkv, bytes] and device tensors; every other dimension is larger than its neighbours."""
    x = bf16_round((rng.standard_normal((n_tiles, c.B, c.Hkv, c.TK, c.Dh)) * std * (1 + 2 * (np.arange(c.Dh) % 2)) * 2.0 ** exp).astype(np.float32))
    host = kv_q4.pages(*kv_q4.quantise(x, exp))
    return host, [torch.from_numpy(t).to(DEV) for t in host]


def decoded(host, c, exp):
    """[B, Hkv, positions, Dh] in 64 bits."""
    v = kv_q4.values(*kv_q4.split(host, c.TK, c.Dh), exp)
    return np.moveaxis(v, 0, 2).reshape(c.B, c.Hkv, -1, c.Dh)


def scratch_for(c, S):
    n = tb.k_attn_q4_scratch_bytes(c, S)
    t = torch.empty(n + 64, dtype=torch.uint8, device=DEV)
    t[n:] = 77                                             # nothing may be written behind it
    t[:n] = 0xff                                           # NaN: nothing of it is read before it is written
    return t, n


def within(got, want, mean, most, sums, p_half):
    """What attention may be off by, relative to the weighted mean of |V|: the weights' rounding for the second product (p_half), the output's (half a bf16 step of
    the value), the score's sum in fp32 - at most 40 additions, of which the tensor cores truncate, so a step of 2^-23 each, of the largest sum of
    |q k|, which moves a weight by as much, in the numerator and in the denominator - and 2^-20 for exponentials and the sums of the weights.
    Weights in fp16 (p_half says so) have an end, too: below 2^-14 they are multiples of 2^-24, off by 2^-25 at most.  The largest is 2^6 at least, where the reference has
    moved, and so is their sum: the result is off by 2^-31 of the sum of |V| over the keys."""
    rel = p_half + 2 * 40 * 2.0 ** -23 * most[..., None] + 2.0 ** -20
    tol = HALF_BF16 * np.abs(want) * (1 + rel) + rel * mean + 1e-30 + (2.0 ** -31 * sums if p_half == HALF_FP16 else 0.0)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(got - want).max(), (np.abs(got - want) / tol).max())


# ---- append and read back ----

def run_append(c, B, S, pos0, k_exp, v_exp, q, k, v, pos=None, tiles=None, seed=5):
    rng = np.random.default_rng(seed)
    n_tiles = (c.max_len + c.TK - 1) // c.TK
    nbytes = tb.k_kv_q4_tile_bytes(c)
    if tiles is None:
        tiles = rng.integers(0, 256, (2, n_tiles, nbytes), dtype=np.uint8)
    kt, vt = ([torch.from_numpy(t.copy()).to(DEV) for t in side] for side in tiles)
    cos, sin = (torch.empty(c.max_len, c.Dh // 2, device=DEV) for _ in range(2))
    tb.k_rope_tables(c.Dh, c.max_len, 10000.0, cos, sin)
    qb = torch.full((B * S, c.Hq * c.Dh), 7.0, dtype=torch.bfloat16, device=DEV)
    dev = [torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DEV) for x in (q, k, v)]
    p = None if pos is None else torch.tensor(pos, dtype=torch.int32, device=DEV)
    tb.k_rope_kv_q4(*dev, qb, kt, vt, cos, sin, c, B, S, pos0, k_exp, v_exp, p)
    kb, vb = (torch.full((B, c.Hkv, S, c.Dh), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    tb.k_kv_unpack_q4(kt, vt, kb, vb, c, B, S, pos0, k_exp, v_exp, p)
    torch.cuda.synchronize()
    after = [np.stack([t.cpu().numpy() for t in side]) for side in (kt, vt)]
    return tiles, after, f32(qb), f32(kb), f32(vb), cos.cpu().numpy(), sin.cpu().numpy()


def check_append(c, B, S, pos0, k_exp, v_exp, q, k, v, pos=None):
    tiles, after, qb, kb, vb, cos, sin = run_append(c, B, S, pos0, k_exp, v_exp, q, k, v, pos)
    want = [t.reshape(len(t), c.B, c.Hkv, -1).copy() for t in tiles]
    q, k, v = (x.reshape(B, S, -1, c.Dh) for x in (q, k, v))
    for b in range(B):
        first = pos0 if pos is None else pos[b]
        if not 0 <= first <= pos0:
            assert (qb.reshape(B, S, -1)[b] == 7).all() and (kb[b] == 7).all() and (vb[b] == 7).all()
            continue
        for t in range(S):
            at = first + t
            rot = lambda x: kv_q4.rotate(x[b, t], cos[at], sin[at])                                    # noqa: E731
            assert np.array_equal(qb.reshape(B, S, c.Hq, c.Dh)[b, t], rot(q), equal_nan=True)
            for side, x, exp, back in ((0, rot(k), k_exp, kb), (1, bf16_round(v[b, t].astype(np.float32)), v_exp, vb)):
                codes, scales = kv_q4.quantise(x, exp)
                page, slot, cut = want[side][at // c.TK, b], at % c.TK, c.TK * c.Dh // 2
                page[:, slot * c.Dh // 2:(slot + 1) * c.Dh // 2] = codes
                page[:, cut + slot * c.Dh // 16:cut + (slot + 1) * c.Dh // 16] = scales
                assert np.array_equal(back[b, :, t], kv_q4.values(codes, scales, exp), equal_nan=True)
    for side in (0, 1):
        assert np.array_equal(after[side].reshape(want[side].shape), want[side])      # the positions, bit for bit, and nothing else


@pytest.mark.parametrize("Hq,Hkv,Dh,TK,B,cB,S,pos0,k_exp,v_exp", [
    (8, 2, 64, 16, 1, 1, 1, 0, 0, 0), (8, 2, 128, 32, 2, 2, 1, 31, 0, -2), (4, 4, 64, 32, 3, 5, 7, 29, 3, -3), (71, 1, 64, 16, 2, 2, 3, 15, 0, 0),
    (32, 8, 128, 256, 1, 1, 300, 100, 0, 0), (3, 1, 128, 48, 2, 3, 50, 40, -32, 32), (1, 1, 64, 16, 1, 1, 33, 0, 32, -32)])
def test_append_gives_the_bits_of_the_definition(Hq, Hkv, Dh, TK, B, cB, S, pos0, k_exp, v_exp):
    rng = np.random.default_rng(Hq * 100 + S)
    c = config(Hq, Hkv, Dh, cB, pos0 + S + 3, TK)
    q, k, v = (rng.standard_normal((B * S, H * Dh)).astype(np.float32) * 2.0 ** e for H, e in ((Hq, 0), (Hkv, k_exp), (Hkv, v_exp)))
    check_append(c, B, S, pos0, k_exp, v_exp, q, k, v)


@pytest.mark.parametrize("pos", [[0, 31, 32, 70], [-1, 70, 71, 5], [2147483647, -2147483648, 0, 1]])
def test_append_at_positions_of_the_sequences_own(pos):
    rng = np.random.default_rng(3)
    c = config(B=4, max_len=96)
    check_append(c, 4, 1, 70, 0, 0, *(rng.standard_normal((4, H * 64)).astype(np.float32) for H in (8, 2, 2)), pos=pos)


def test_append_of_values_at_borders_and_ends():
    """Borders of codes and of scales, values that round to nothing, beyond the largest, subnormal, infinite and NaN; position 0 does not rotate."""
    c = config(Hq=2, Hkv=2, Dh=64, B=1, max_len=16, TK=16)
    borders = np.array([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, -0.0], np.float32)
    rows = [np.concatenate([borders * s for s in (1.0, 1.125, 2.0 ** -9, 448.0)]),
            np.concatenate([np.full(16, x) for x in (6 * 2.0 ** -10, 6 * 2.0 ** -10 * (1 + 2.0 ** -7), 6 * 464.0, 3.0e38)]),
            np.concatenate([np.full(16, x) for x in (6 * 1.0625, 6 * 1.1875, 1e-38, 1e-45)]),
            np.concatenate([np.zeros(16), [np.inf] + [1.0] * 15, [np.nan] * 16, [1.0] * 15 + [-np.inf]]),
            np.concatenate([np.full(16, -0.0), np.full(16, 3.4e38), np.full(16, -1.0), borders[::-1]])]
    for row in rows:
        x = np.tile(row.astype(np.float32), 2).reshape(1, -1)
        for k_exp, v_exp in ((0, 0), (-32, 32), (5, -7)):
            check_append(c, 1, 1, 0, k_exp, v_exp, np.ones((1, 128), np.float32), x, x)


def test_rotation_is_that_of_exact_sums():
    """Products that cancel: without their low parts the difference has none of its bits right."""
    c = config(Hq=4, Hkv=2, Dh=64, B=1, max_len=64, TK=16)
    rng = np.random.default_rng(9)
    q = rng.standard_normal((40, 4, 64))
    ang = np.arange(40)[:, None] * 10000.0 ** (-np.arange(32) / 32)
    q[:, :, 32:] = q[:, :, :32] / np.tan(np.where(np.sin(ang) == 0, 1, ang))[:, None]            # lo cos = hi sin, up to rounding
    q[0] = 1
    check_append(c, 1, 40, 0, 0, 0, q.reshape(40, -1).astype(np.float32), rng.standard_normal((40, 128)).astype(np.float32), rng.standard_normal((40, 128)).astype(np.float32))


def test_rotation_rounds_to_fp32_and_then_to_bf16():
    """Sums that fp32 rounds to the middle of two bf16 numbers go to the even one, whichever side they came from; those that it does not, to the nearer."""
    c = config(Hq=2, Hkv=1, Dh=64, B=1, max_len=16, TK=16)
    rest = np.array([2.0 ** -30, -2.0 ** -30, 2.0 ** -24, -2.0 ** -24, 2.0 ** -23, -2.0 ** -23, 0, 2.0 ** -60])
    one = np.resize([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8], 32)              # the middles between 1, 1 + 2^-7 and 1 + 2^-6
    row = np.concatenate((one, np.repeat(rest, 4))).astype(np.float32)
    cos, sin = (torch.full((16, 32), x, device=DEV) for x in (1.0, -1.0))
    x = torch.from_numpy(np.tile(row, 4)).to(DEV)
    qb, tiles = torch.empty(1, 128, dtype=torch.bfloat16, device=DEV), [torch.zeros(tb.k_kv_q4_tile_bytes(c), dtype=torch.uint8, device=DEV) for _ in range(2)]
    tb.k_rope_kv_q4(x[:128], x[128:192], x[192:], qb, tiles[:1], tiles[1:], cos, sin, c, 1, 1, 0)
    got = f32(qb).reshape(2, 64)
    assert np.array_equal(got[0], got[1]) and np.array_equal(got[0], kv_q4.rotate(row, np.float32(1), np.float32(-1)))
    assert list(got[0, :4]) == [1, 1 + 2.0 ** -6] * 2 and list(got[0, 16:24]) == [1 + 2.0 ** -7, 1 + 2.0 ** -6] * 2 + [1, 1 + 2.0 ** -7] * 2


# ---- attention ----

def run_attn(c, B, S, pos0, q, kt, vt, k_exp=0, v_exp=0, pos=None, stream=None):
    qb, ob = bf16(q.reshape(B * S, -1)), torch.full((B * S + 1, c.Hq * c.Dh), 7.0, dtype=torch.bfloat16, device=DEV)
    s, n = scratch_for(c, S)
    p = None if pos is None else torch.tensor(pos, dtype=torch.int32, device=DEV)
    tb.k_attn_q4(qb, kt, vt, ob, c, B, S, pos0, k_exp, v_exp, p, s, stream)
    torch.cuda.synchronize()
    assert (s[n:] == 77).all() and (ob[B * S] == 7).all()
    return f32(ob)[:B * S].reshape(B, S, c.Hq, c.Dh)


def check_attn(c, B, S, pos0, k_exp=0, v_exp=0, pos=None, seed=1, std_q=1.0, p_half=HALF_FP16, change=None):
    rng = np.random.default_rng(seed)
    n_tiles = (pos0 + S + c.TK - 1) // c.TK
    (kh, kt), (vh, vt) = random_tiles(rng, c, n_tiles, k_exp), random_tiles(rng, c, n_tiles, v_exp)
    q = bf16_round((rng.standard_normal((B, S, c.Hq, c.Dh)) * std_q * 2.0 ** -k_exp).astype(np.float32))
    if change:
        change(q, kh, vh)
        kt, vt = ([torch.from_numpy(t).to(DEV) for t in side] for side in (kh, vh))
    got = run_attn(c, B, S, pos0, q, kt, vt, k_exp, v_exp, pos)
    K, V = decoded(kh, c, k_exp), decoded(vh, c, v_exp)
    for b in range(B):
        first = pos0 if pos is None else pos[b]
        if not 0 <= first <= pos0:
            assert (got[b] == 0).all()
            continue
        within(got[b], *kv_q4.attention(q[b].astype(np.float64), K[b], V[b], first), p_half)
    return q, kh, vh, got


@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 7, 8, 16])
@pytest.mark.parametrize("pos0", [0, 1, 14, 15, 16, 17, 63, 64, 200])
def test_single_tokens(Dh, G, pos0):
    c = config(2 * G, 2, Dh, 2, 256, 32)
    check_attn(c, 2, 1, pos0, seed=pos0)


@pytest.mark.parametrize("Dh,G,Hkv,B,cB,S,pos0,TK", [
    (64, 4, 2, 1, 1, 2, 0, 16), (128, 4, 2, 2, 3, 5, 100, 32), (64, 1, 1, 3, 3, 9, 3, 16), (128, 8, 1, 1, 1, 8, 15, 16), (64, 3, 2, 2, 2, 21, 30, 32), (128, 2, 2, 1, 1, 32, 0, 48),
    (128, 16, 1, 2, 2, 4, 60, 64), (64, 64, 1, 1, 1, 1, 40, 16), (64, 71, 1, 2, 2, 1, 90, 32), (128, 8, 2, 1, 1, 3, 700, 256)])
def test_a_few_tokens(Dh, G, Hkv, B, cB, S, pos0, TK):
    check_attn(config(G * Hkv, Hkv, Dh, cB, pos0 + S, TK), B, S, pos0, seed=S)


@pytest.mark.parametrize("Dh,G,Hkv,B,S,pos0,TK", [
    (64, 4, 2, 2, 17, 0, 16), (128, 4, 1, 1, 40, 77, 32), (64, 1, 2, 1, 65, 3, 16), (128, 8, 1, 2, 130, 0, 32), (64, 2, 2, 1, 200, 50, 48), (128, 4, 2, 1, 129, 300, 256), (64, 71, 1, 1, 2, 33, 16),
                                                  (128, 1, 2, 1, 200, 500, 64), (64, 8, 2, 3, 127, 40, 32), (64, 8, 2, 6, 150, 0, 64)])
def test_prompts(Dh, G, Hkv, B, S, pos0, TK):
    check_attn(config(G * Hkv, Hkv, Dh, B, pos0 + S, TK), B, S, pos0, seed=S, p_half=HALF_FP16 if S < 128 else HALF_BF16)


UNPACKED = [(64, 8, 4, 3, 127, 700, 64), (128, 4, 8, 6, 64, 601, 48), (128, 8, 8, 8, 33, 500, 128), (64, 1, 16, 8, 100, 200, 16), (64, 8, 8, 1, 200, 300, 32)]


@pytest.mark.parametrize("Dh,G,Hkv,B,S,pos0,TK", UNPACKED)
def test_queries_enough_to_unpack_the_cache_for(Dh, G, Hkv, B, S, pos0, TK):
    """From 32 queries on, where that is expected to be faster: the scratch array then holds the keys as bf16 (weights are bf16 numbers, too)."""
    c = config(G * Hkv, Hkv, Dh, B, pos0 + S, TK)
    rng = np.random.default_rng(S)
    n_tiles = (pos0 + S + TK - 1) // TK
    (kh, kt), (vh, vt) = random_tiles(rng, c, n_tiles, 1), random_tiles(rng, c, n_tiles, -1)
    q = bf16_round((rng.standard_normal((B, S, c.Hq, Dh)) / 2).astype(np.float32))
    qb, ob = bf16(q.reshape(B * S, -1)), torch.full((B * S + 1, c.Hq * Dh), 7.0, dtype=torch.bfloat16, device=DEV)
    s, n = scratch_for(c, S)
    tb.k_attn_q4(qb, kt, vt, ob, c, B, S, pos0, 1, -1, None, s)
    torch.cuda.synchronize()
    assert (s[n:] == 77).all() and (ob[B * S] == 7).all()
    K, V = decoded(kh, c, 1), decoded(vh, c, -1)
    assert np.array_equal(f32(s[:2 * Dh * pos0].view(torch.bfloat16)).reshape(pos0, Dh), K[0, 0, :pos0])
    got = f32(ob)[:B * S].reshape(B, S, c.Hq, Dh)
    for b in range(B):
        within(got[b], *kv_q4.attention(q[b].astype(np.float64), K[b], V[b], pos0), HALF_BF16)


@pytest.mark.parametrize("Dh,G,Hkv,B,S,pos0,TK", UNPACKED)
@pytest.mark.parametrize("side", ["k", "v"])
def test_a_nan_in_a_cache_that_is_unpacked(Dh, G, Hkv, B, S, pos0, TK, side):
    """A group of the last sequence stands for NaN at one of the call's own positions: of its head's outputs those that see it, and no other."""
    c = config(G * Hkv, Hkv, Dh, B, pos0 + S, TK)
    at, group, head = pos0 + S // 2, 2, 1
    rng = np.random.default_rng(S + 1)
    n_tiles = (pos0 + S + TK - 1) // TK
    (kh, _), (vh, _) = random_tiles(rng, c, n_tiles, 0), random_tiles(rng, c, n_tiles, 0)
    t = kh if side == "k" else vh
    t[at // TK, B - 1, head, TK * Dh // 2 + (at % TK) * Dh // 16 + group] = 0x7f
    got = run_attn(c, B, S, pos0, bf16_round(rng.standard_normal((B, S, c.Hq, Dh)).astype(np.float32)), *([torch.from_numpy(x).to(DEV) for x in y] for y in (kh, vh)))
    nan = np.zeros(got.shape, bool)
    nan[B - 1, S // 2:, head * G:(head + 1) * G] = True
    if side == "v":
        nan[..., :16 * group] = nan[..., 16 * (group + 1):] = False
    assert np.array_equal(np.isnan(got), nan)


@pytest.mark.parametrize("B,pos0,Hq,Hkv,Dh,TK", [(1, 4000, 8, 2, 128, 128), (1, 16383, 4, 1, 64, 256), (2, 1023, 8, 8, 64, 16), (40, 130, 16, 4, 128, 16), (300, 33, 8, 8, 64, 48)])
def test_contexts_in_parts_and_in_one(B, pos0, Hq, Hkv, Dh, TK):
    """One sequence of a long context is split over the GPU; many sequences of a short one are not."""
    check_attn(config(Hq, Hkv, Dh, B, pos0 + 1, TK), B, 1, pos0)


@pytest.mark.parametrize("pos", [[0, 15, 16, 299, 120], [-1, 300, 299, -5, 17], [-1, -1, -1, -1, -1], [2147483647, 0, 1, 2, -2147483648]])
@pytest.mark.parametrize("Dh,G", [(64, 4), (128, 16)])
def test_positions_of_the_sequences_own(pos, Dh, G):
    check_attn(config(2 * G, 2, Dh, 5, 300, 16 if Dh == 64 else 64), 5, 1, 299, pos=pos)


@pytest.mark.parametrize("k_exp,v_exp", [(32, -32), (-32, 32), (3, -2)])
def test_exponents(k_exp, v_exp):
    check_attn(config(8, 2, 128, 1, 80, 16), 1, 1, 70, k_exp, v_exp)
    check_attn(config(8, 2, 64, 1, 80, 16), 1, 33, 40, k_exp, v_exp, p_half=HALF_BF16)


@pytest.mark.parametrize("std_q", [2.0 ** -100, 1e-6, 30.0, 400.0])
def test_queries_of_any_size(std_q):
    """fp16 would hold neither the smallest nor the largest; large ones leave a few keys with all of the weight, wherever they lie."""
    for S in (1, 6):
        check_attn(config(8, 2, 128, 2, 700, 64), 2, S, 600, std_q=std_q)


@pytest.mark.parametrize("above,S,pos0", [(10, 1, 200), (17, 1, 200), (17, 5, 90), (18, 1, 200), (18, 5, 90)])
def test_queries_whose_numbers_are_far_apart(above, S, pos0):
    """One dimension of each query is 2^above times the others, and zero in the keys.  As fp16, scaled by the largest, the others are exact down to 2^-17 of it; below they
    are off by 2^-25 of it, a score d by as much of the sum of |k|, and its weight by a factor of exp(d), as the sum of the weights."""
    c, n = config(8, 2, 64, 2, 256, 32), pos0 + S
    rng = np.random.default_rng(above)
    (kh, _), (vh, vt) = random_tiles(rng, c, 8, 0), random_tiles(rng, c, 8, 0)
    kh[..., 5:32 * 32:32] &= 0xf0                          # codes of dimension 10
    q = rng.choice([-1, 1], (2, S, 8, 64)) * (1 + rng.integers(0, 128, (2, S, 8, 64)) / 128)
    q[..., 10] = 2.0 ** above
    got = run_attn(c, 2, S, pos0, q, [torch.from_numpy(t).to(DEV) for t in kh], vt)
    K, V = decoded(kh, c, 0), decoded(vh, c, 0)
    assert not K[..., 10].any()
    for b in range(2):
        d = 2.0 ** (above - 25) * np.abs(K[b, :, :n]).sum(-1).max() / 8 if above > 17 else 0.0
        within(got[b], *kv_q4.attention(q[b], K[b], V[b], pos0), HALF_FP16 + np.expm1(2 * d) if d else HALF_FP16)


def test_scores_that_rise_with_every_key():
    """The largest score so far is always the last: the reference moves again and again."""
    def change(q, kh, vh):
        q[:] = np.abs(q)
        c_codes, c_scales = kv_q4.split(kh, 32, 128)
        c_codes[:] = 0x22                                  # 1, 1
        for j in range(len(kh)):
            c_scales[j] = (0x20 + j * 8 + np.arange(32)[:, None] // 8)                # rising scales
        kh[:] = kv_q4.pages(c_codes, c_scales)
    check_attn(config(8, 2, 128, 1, 256, 32), 1, 1, 255, change=change)
    check_attn(config(8, 2, 128, 1, 256, 32), 1, 8, 248, change=change)


@pytest.mark.parametrize("S,pos0", [(1, 37), (1, 47), (5, 20), (5, 43), (40, 3)])
def test_what_lies_behind_the_sequence_is_not_read(S, pos0):
    """Codes, scales and NaN of positions that no query sees, in the same chunk and the same tile."""
    c = config(8, 2, 64, 2, 64, 32)
    def change(q, kh, vh):
        for t in (kh, vh):
            codes, scales = kv_q4.split(t, 32, 64)
            for j in range(len(t)):
                for s in range(32):
                    if j * 32 + s >= pos0 + S:
                        codes[j, :, :, s], scales[j, :, :, s] = 0xff, 0x7f if s % 2 else 0xff
            t[:] = kv_q4.pages(codes, scales)
    check_attn(c, 2, S, pos0, change=change)


@pytest.mark.parametrize("Dh,G,S,pos0,TK", [(64, 4, 5, 30, 16), (128, 4, 16, 10, 32), (64, 1, 9, 0, 16), (128, 2, 30, 3, 16),
                                              (64, 4, 20, 30, 16), (128, 4, 70, 10, 32), (64, 2, 200, 40, 64), (128, 8, 130, 0, 16)])
@pytest.mark.parametrize("side", ["k", "v"])
def test_a_nan_reaches_the_queries_that_see_it_and_no_other(Dh, G, S, pos0, TK, side):
    """A group of a key or value stands for NaN at one of the call's own positions, which earlier queries do not see."""
    c = config(2 * G, 2, Dh, 1, pos0 + S, TK)
    at, group, head = pos0 + S // 2, 1, 1
    rng = np.random.default_rng(4)
    n_tiles = (pos0 + S + TK - 1) // TK
    (kh, _), (vh, _) = random_tiles(rng, c, n_tiles, 0), random_tiles(rng, c, n_tiles, 0)
    q = bf16_round(rng.standard_normal((1, S, 2 * G, Dh)).astype(np.float32))
    clean = run_attn(c, 1, S, pos0, q, *([torch.from_numpy(t).to(DEV) for t in s] for s in (kh, vh)))
    K, V = decoded(kh, c, 0)[0], decoded(vh, c, 0)[0]
    t = kh if side == "k" else vh
    t[at // TK, 0, head, TK * Dh // 2 + (at % TK) * Dh // 16 + group] = 0x7f
    got = run_attn(c, 1, S, pos0, q, *([torch.from_numpy(t).to(DEV) for t in s] for s in (kh, vh)))
    nan = np.zeros(got.shape, bool)
    nan[0, S // 2:, head * G:] = True
    if side == "v":
        nan[..., :16 * group] = nan[..., 16 * (group + 1):] = False
    assert np.array_equal(np.isnan(got), nan)
    if S < 128:
        assert np.array_equal(got[~nan], clean[~nan])
    else:                                                  # (a NaN moves the reference of the rows of its warp: other bits, by what any reference may differ)
        want = kv_q4.attention(q[0].astype(np.float64), K, V, pos0)
        within(np.where(nan, want[0], got)[0], *want, HALF_BF16)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_queries_that_are_not_finite_give_nan(bad):
    c = config(8, 2, 64, 2, 64, 32)
    rng = np.random.default_rng(2)
    (_, kt), (_, vt) = random_tiles(rng, c, 2, 0), random_tiles(rng, c, 2, 0)
    q = rng.standard_normal((2, 1, 8, 64)).astype(np.float32)
    q[1, 0, 3, 10] = bad
    got = run_attn(c, 2, 1, 40, q, kt, vt)
    nan = np.zeros(got.shape, bool)
    nan[1, 0, 3] = True
    assert np.array_equal(np.isnan(got), nan)


def test_zero_keys_give_the_mean():
    c = config(8, 2, 128, 1, 64, 16)
    check_attn(c, 1, 1, 60, change=lambda q, kh, vh: kh.fill(0))


def test_a_shrunken_batch_uses_the_tiles_of_the_whole():
    """Two of five sequences; tiles behind the positions may be missing."""
    rng = np.random.default_rng(6)
    c = config(8, 2, 64, 5, 512, 32)
    (kh, kt), (vh, vt) = random_tiles(rng, c, 3, 0), random_tiles(rng, c, 3, 0)
    q = bf16_round(rng.standard_normal((2, 1, 8, 64)).astype(np.float32))
    got = run_attn(c, 2, 1, 70, q, kt + [None] * 13, vt + [None] * 13)
    for b in range(2):
        within(got[b], *kv_q4.attention(q[b].astype(np.float64), decoded(kh, c, 0)[b], decoded(vh, c, 0)[b], 70), HALF_FP16)


def test_offsets_that_pass_32_bits():
    """A tile of more than 4 GB: the last sequence's page lies behind 2^32 bytes of it."""
    c = config(8, 8, 128, 1900, 4096, 4096)
    nbytes = tb.k_kv_q4_tile_bytes(c)
    assert nbytes > 1 << 32
    rng = np.random.default_rng(8)
    one = config(8, 8, 128, 1, 4096, 4096)
    (kh, _), (vh, _) = random_tiles(rng, one, 1, 0), random_tiles(rng, one, 1, 0)
    tiles = []
    for h in (kh, vh):
        t = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)
        t[-h.size:] = torch.from_numpy(h.reshape(-1)).to(DEV)
        tiles.append([t])
    pos = np.full(1900, -1, np.int32)
    pos[1899] = 4000
    q = bf16_round(rng.standard_normal((1900, 1, 8, 128)).astype(np.float32))
    qb, ob = bf16(q.reshape(1900, -1)), torch.full((1900, 1024), 7.0, dtype=torch.bfloat16, device=DEV)
    s, _ = scratch_for(c, 1)
    tb.k_attn_q4(qb, *tiles, ob, c, 1900, 1, 4000, 0, 0, torch.from_numpy(pos).to(DEV), s)
    got = f32(ob).reshape(1900, 1, 8, 128)
    assert (got[:1899] == 0).all()
    within(got[1899], *kv_q4.attention(q[1899].astype(np.float64), decoded(kh, one, 0)[0], decoded(vh, one, 0)[0], 4000), HALF_FP16)
    new = [torch.randn(1900, H * 128, device=DEV, generator=torch.Generator(DEV).manual_seed(1)) for H in (8, 8, 8)]
    cos, sin = (torch.empty(4096, 64, device=DEV) for _ in range(2))
    tb.k_rope_tables(128, 4096, 10000.0, cos, sin)
    tb.k_rope_kv_q4(*new, qb, *tiles, cos, sin, c, 1900, 1, 4000, 0, 0, torch.from_numpy(pos).to(DEV))
    kb, vb = (torch.zeros(1900, 8, 1, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    tb.k_kv_unpack_q4(*tiles, kb, vb, c, 1900, 1, 4000, 0, 0, torch.from_numpy(pos).to(DEV))
    want = kv_q4.values(*kv_q4.quantise(bf16_round(new[2][1899].cpu().numpy().reshape(8, 128)), 0), 0)
    assert np.array_equal(f32(vb)[1899, :, 0], want) and not vb[:1899].any()
    tb.k_kv_move(*tiles, [1899], [1898], c, tb.KV_Q4, 1900, 4001)
    tb.k_kv_unpack_q4(*tiles, kb, vb, c, 1900, 1, 4000, 0, 0, torch.from_numpy(np.where(np.arange(1900) == 1898, 4000, -1).astype(np.int32)).to(DEV))
    assert np.array_equal(f32(vb)[1898, :, 0], want)


@pytest.mark.parametrize("B,S,Hq,Dh", [(9, 128, 16, 128), (11, 64, 64, 128), (17, 130, 16, 64)])
def test_a_cache_that_is_unpacked_in_groups_of_sequences(B, S, Hq, Dh):
    """Sequences of 131072 positions, more than the scratch array holds as bf16: each group's outputs are those of a call of its own, with a NaN in one of its values."""
    n, Hkv, TK = 131072, 8, 2048
    c, pos0 = config(Hq, Hkv, Dh, B, n, TK), n - S
    g = torch.Generator(DEV).manual_seed(B)
    tiles = []
    for _ in range(2):
        t = torch.randint(0, 256, (n // TK, B, Hkv, TK * Dh * 9 // 16), dtype=torch.uint8, device=DEV, generator=g)
        t[..., TK * Dh // 2:] = torch.randint(0x28, 0x38, t[..., TK * Dh // 2:].shape, dtype=torch.uint8, device=DEV, generator=g)
        tiles.append(t)
    tiles[1][(n - S // 2) // TK, B - 1, 3, TK * Dh // 2 + (n - S // 2) % TK * Dh // 16 + 1] = 0x7f      # seen by the last sequence's later queries
    qb = torch.randn(B * S, Hq * Dh, device=DEV, generator=g).bfloat16()
    ob = torch.full((B * S + 1, Hq * Dh), 7.0, dtype=torch.bfloat16, device=DEV)
    s, nbytes = scratch_for(c, S)
    fit = nbytes // (2 * Hkv * n * Dh * 2)
    pages = lambda b: [[t[b:].data_ptr() for t in side] for side in tiles]                             # noqa: E731
    assert 1 < fit < B
    tb.k_attn_q4(qb, list(tiles[0]), list(tiles[1]), ob, c, B, S, pos0, 0, 0, None, s)
    groups = -(-B // fit)
    most = -(-B // groups)
    want = torch.empty_like(ob[:B * S])
    for b in range(0, B, most):
        m = min(most, B - b)
        tb.k_attn_q4(qb[b * S:], *pages(b), want[b * S:], c, m, S, pos0, 0, 0, None, s)
    torch.cuda.synchronize()
    assert (s[nbytes:] == 77).all() and (ob[B * S] == 7).all()
    nan = torch.zeros(B, S, Hq, Dh, dtype=torch.bool, device=DEV)
    nan[B - 1, S - S // 2:, 3 * (Hq // Hkv):4 * (Hq // Hkv), 16:32] = True
    assert torch.equal(torch.isnan(ob[:B * S]), nan.view(B * S, -1))
    assert torch.equal(ob[:B * S].nan_to_num(), want.nan_to_num())
    # and the last queries as single ones, which read the codes: |V| is below 3 on average, of which the weights' rounding to bf16 moves an output by half a step, as the
    # outputs' own roundings do, of less than that
    single = torch.empty(1, Hq * Dh, dtype=torch.bfloat16, device=DEV)
    one, _ = scratch_for(c, 1)
    for b in (0, most, B - 2):
        tb.k_attn_q4(qb[(b + 1) * S - 1:], *pages(b), single, c, 1, 1, n - 1, 0, 0, None, one)
        assert (single[0].float() - ob[(b + 1) * S - 1].float()).abs().max() <= 2 * HALF_BF16 * 3


def test_two_calls_at_once_on_two_streams():
    c = config(32, 8, 128, 2, 4096, 128)
    rng = np.random.default_rng(7)
    streams = [torch.cuda.Stream(DEV) for _ in range(2)]
    jobs = []
    for s in streams:
        (kh, kt), (vh, vt) = random_tiles(rng, c, 32, 0), random_tiles(rng, c, 32, 0)
        q = bf16(rng.standard_normal((2, 32 * 128)))
        ob = torch.empty(2, 32 * 128, dtype=torch.bfloat16, device=DEV)
        want = torch.empty_like(ob)
        scratch, _ = scratch_for(c, 1)
        tb.k_attn_q4(q, kt, vt, want, c, 2, 1, 4000, 0, 0, None, scratch)
        jobs.append((q, kt, vt, ob, want, scratch))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (q, kt, vt, ob, _, scratch) in zip(streams, jobs):
            tb.k_attn_q4(q, kt, vt, ob, c, 2, 1, 4000, 0, 0, None, scratch, s)
    torch.cuda.synchronize()
    for *_, ob, want, _ in jobs:
        assert torch.equal(ob, want)


def test_a_captured_step_is_replayed_at_other_positions():
    """Append, attention and sampling of one token, captured once: positions, random numbers and inputs are read at every replay."""
    B, c = 3, config(8, 2, 64, 3, 128, 32)
    rng = np.random.default_rng(11)
    (kh, kt), (vh, vt) = random_tiles(rng, c, 4, 0), random_tiles(rng, c, 4, 0)
    cos, sin = (torch.empty(128, 32, device=DEV) for _ in range(2))
    tb.k_rope_tables(64, 128, 10000.0, cos, sin)
    new = [torch.empty(B, H * 64, device=DEV) for H in (8, 2, 2)]
    qb, ob = (torch.empty(B, 512, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pos, u, token = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    scratch, _ = scratch_for(c, 1)
    logits = torch.empty(B, 512, device=DEV)

    def step(stream):
        tb.k_rope_kv_q4(*new, qb, kt, vt, cos, sin, c, B, 1, 127, 0, 0, pos, stream)
        tb.k_attn_q4(qb, kt, vt, ob, c, B, 1, 127, 0, 0, pos, scratch, stream)
        logits.copy_(ob)
        tb.k_sample(logits, u, token, B, 512, None, None, None, None, stream)

    s = torch.cuda.Stream(DEV)
    with torch.cuda.stream(s):
        step(s)                                            # (function attributes)
    torch.cuda.synchronize()
    for t, h in zip(kt + vt, list(kh) + list(vh)):
        t.copy_(torch.from_numpy(h))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(torch.cuda.current_stream())
    for at in ([5, 40, -1], [6, 41, 90], [127, 0, 91]):
        x = [rng.standard_normal(t.shape).astype(np.float32) for t in new]
        for t, v in zip(new, x):
            t.copy_(torch.from_numpy(v))
        pos.copy_(torch.tensor(at, dtype=torch.int32))
        u.copy_(torch.from_numpy(rng.random(B).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            if at[b] < 0:
                assert not ob[b].any()
                continue
            cs, sn = cos.cpu().numpy()[at[b]], sin.cpu().numpy()[at[b]]
            q = kv_q4.rotate(x[0][b].reshape(8, 64), cs, sn)
            for h, v in ((kh, kv_q4.rotate(x[1][b].reshape(2, 64), cs, sn)), (vh, bf16_round(x[2][b].reshape(2, 64)))):
                codes, scales = kv_q4.split(h, 32, 64)
                codes[at[b] // 32, b, :, at[b] % 32], scales[at[b] // 32, b, :, at[b] % 32] = kv_q4.quantise(v, 0)
                h[:] = kv_q4.pages(codes, scales)
            within(f32(ob)[b].reshape(1, 8, 64), *kv_q4.attention(q[None].astype(np.float64), decoded(kh, c, 0)[b], decoded(vh, c, 0)[b], at[b]), HALF_FP16)
            assert int(token[b]) == sample.sample(f32(logits)[b], float(u[b]))
    for t, h in zip(kt + vt, list(kh) + list(vh)):
        assert np.array_equal(t.cpu().numpy(), h)


# ---- moves ----

def maps(rng, B):
    some = lambda n: list(rng.choice(B, size=n, replace=False))           # noqa: E731
    ring = some(min(B, 7))
    yield [(0, b) for b in range(1, B)]                                   # one for all
    yield list(zip(range(B), rng.permutation(B)))                         # any permutation
    yield list(zip(ring, ring[1:] + ring[:1]))                            # a cycle
    yield list(zip(ring, ring[1:])) + [(ring[0], ring[0])]                # a chain, and a place that takes itself
    yield [(-1, b) for b in some((B + 1) // 2)]                           # freed
    dst = some(B)
    yield [(int(rng.integers(-1, B)), b) for b in dst]                    # any map at all
    yield list(zip(range(B - B // 3, B), range(B // 3)))                  # the last ones into the first places


@pytest.mark.parametrize("form,Dh,Hkv,TK,B,n_tiles,length", [
    (tb.KV_Q4, 64, 2, 16, 5, 3, 40), (tb.KV_Q4, 128, 1, 32, 9, 1, 1), (tb.KV_Q4, 128, 3, 48, 4, 2, 96), (tb.KV_BF16, 64, 2, 4, 6, 5, 18), (tb.KV_BF16, 8, 3, 7, 11, 2, 9),
    (tb.KV_BF16, 128, 8, 64, 3, 2, 65), (tb.KV_Q4, 64, 1, 16, 300, 1, 13), (tb.KV_BF16, 16, 1, 5, 700, 1, 5), (tb.KV_BF16, 64, 1, 16, 2, 4, 64), (tb.KV_Q4, 64, 8, 256, 2, 2, 300)])
def test_moves_of_every_kind(form, Dh, Hkv, TK, B, n_tiles, length):
    rng = np.random.default_rng(B)
    c = config(Hkv, Hkv, Dh, B, n_tiles * TK, TK)
    widths = [Dh // 2, Dh // 16] if form == tb.KV_Q4 else [2 * Dh]
    before = rng.integers(0, 256, (2, n_tiles, B, Hkv, TK * sum(widths)), dtype=np.uint8)
    for pairs in maps(rng, B):
        pairs = [(int(a), int(b)) for a, b in pairs]
        sides = [[torch.from_numpy(t.copy()).to(DEV) for t in s] for s in before]
        tb.k_kv_move(*sides, [a for a, _ in pairs], [b for _, b in pairs], c, form, B, length)
        torch.cuda.synchronize()
        for side, s in zip(sides, before):
            assert np.array_equal(np.stack([t.cpu().numpy() for t in side]), kv_q4.moved(s, pairs, TK, length, widths)), pairs


# ---- together ----

def test_a_prompt_forked_into_sampled_answers():
    """A model of one layer: a prompt in one place, forked into the others, answers sampled token by token at positions of their own, finished ones compacted away.
    Every step is checked from what the GPU had before it."""
    B, V, TK, S, c = 6, 512, 16, 37, config(8, 2, 64, 6, 96, 16)
    rng = np.random.default_rng(21)
    d = 512
    W = {n: bf16_round((rng.standard_normal((rows, d)) * d ** -0.5).astype(np.float32)) for n, rows in (("q", 512), ("k", 128), ("v", 128), ("lm", V))}
    embed, gain = bf16_round(rng.standard_normal((V, d)).astype(np.float32)), bf16_round((1 + 0.1 * rng.standard_normal(d)).astype(np.float32))
    Wd, embed_d, gain_d = {n: bf16(w) for n, w in W.items()}, bf16(embed), bf16(gain)
    cos, sin = (torch.empty(96, 32, device=DEV) for _ in range(2))
    tb.k_rope_tables(64, 96, 10000.0, cos, sin)
    n_tiles, nbytes = 6, tb.k_kv_q4_tile_bytes(c)
    kt, vt = ([torch.zeros(nbytes, dtype=torch.uint8, device=DEV) for _ in range(n_tiles)] for _ in range(2))
    settings = [torch.tensor(x, device=DEV) for x in ([0.9, 1.0, 1.3, 0.7, 0.0, 2.0], [0, 40, 7, 0, 3, 100], [1.0, 0.9, 0.8, 0.5, 0.9, 0.95], [0.0, 0.0, 0.05, 0.1, 0.0, 0.02])]
    settings[1] = settings[1].int()

    def forward(tokens, n, S_, pos0, pos):
        """n sequences of S_ tokens; returns logits of every token and what they were computed from."""
        M = n * S_
        tok = torch.tensor(tokens, dtype=torch.int32, device=DEV)
        x, h = torch.empty(M, d, device=DEV), torch.empty(M, d, dtype=torch.bfloat16, device=DEV)
        q, k, v, logits = (torch.empty(M, w, device=DEV) for w in (512, 128, 128, V))
        qb, ob = (torch.empty(M, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        scratch, _ = scratch_for(c, S_)
        tb.k_embed(embed_d, tok, x, M, d, V)
        tb.k_rmsnorm(x, d, gain_d, h, M, d, 1e-5)
        tb.k_gemm_group(h, [Wd["q"], Wd["k"], Wd["v"]], [q, k, v], M, [512, 128, 128], d, [512, 128, 128])
        tb.k_rope_kv_q4(q, k, v, qb, kt, vt, cos, sin, c, n, S_, pos0, 0, 0, pos)
        tb.k_attn_q4(qb, kt, vt, ob, c, n, S_, pos0, 0, 0, pos, scratch)
        tb.k_gemm(ob, Wd["lm"], logits, M, V, d, V, 0, False)
        return logits, dict(q=q.cpu().numpy(), k=k.cpu().numpy(), v=v.cpu().numpy(), o=f32(ob))

    cos_h, sin_h = cos.cpu().numpy(), sin.cpu().numpy()
    host = [np.zeros((n_tiles, B, 2, nbytes // (B * 2)), np.uint8) for _ in range(2)]

    def follow(parts, n, S_, first):
        """The oracle's cache and attention from the GPU's projections; the cache is equal bit for bit."""
        for b in range(n):
            for t in range(S_):
                at, m = int(first[b]) + t, b * S_ + t
                for h, x in ((host[0], kv_q4.rotate(parts["k"][m].reshape(2, 64), cos_h[at], sin_h[at])), (host[1], bf16_round(parts["v"][m].reshape(2, 64)))):
                    codes, scales = kv_q4.split(h, TK, 64)
                    codes[at // TK, b, :, at % TK], scales[at // TK, b, :, at % TK] = kv_q4.quantise(x, 0)
                    h[:] = kv_q4.pages(codes, scales)
            q = np.stack([kv_q4.rotate(parts["q"][b * S_ + t].reshape(8, 64), cos_h[int(first[b]) + t], sin_h[int(first[b]) + t]) for t in range(S_)])
            within(parts["o"][b * S_:(b + 1) * S_].reshape(S_, 8, 64), *kv_q4.attention(q.astype(np.float64), decoded(host[0], c, 0)[b], decoded(host[1], c, 0)[b], int(first[b])),
                   HALF_FP16 if S_ == 1 else HALF_BF16)
        for side, h in ((kt, host[0]), (vt, host[1])):
            assert np.array_equal(np.stack([t.cpu().numpy() for t in side]).reshape(h.shape), h)

    logits, parts = forward(rng.integers(0, V, S), 1, S, 0, None)
    follow(parts, 1, S, [0])
    pairs = [(0, b) for b in range(1, B)]
    tb.k_kv_move(kt, vt, [a for a, _ in pairs], [b for _, b in pairs], c, tb.KV_Q4, B, S)
    for i in range(2):
        host[i] = kv_q4.moved(host[i], pairs, TK, S, [32, 4])
    last = logits[S - 1:S].repeat(B, 1).contiguous()
    live, pos, length = list(range(B)), np.full(B, S), {i: 0 for i in range(B)}
    for step in range(12):
        n = len(live)
        u = rng.random(n).astype(np.float32)
        token = torch.empty(n, dtype=torch.int32, device=DEV)
        mine = [s[torch.tensor(live, device=DEV)].contiguous() for s in settings]
        tb.k_sample(last, torch.from_numpy(u).to(DEV), token, n, V, *mine)
        tokens, rows = token.cpu().numpy(), last.cpu().numpy()
        for i in range(n):
            t, k_, p, m = (float(s[i]) for s in mine)
            assert tokens[i] == sample.sample(rows[i], float(u[i]), t, int(k_), p, m)
            length[live[i]] += 1
        gone = [i for i in range(n) if length[live[i]] >= 3 + 2 * live[i]]           # the answers end at lengths of their own
        if gone:
            keep = [i for i in range(n) if i not in gone]
            holes = [i for i in gone if i < len(keep)]
            pairs = list(zip([i for i in keep if i >= len(keep)], holes))
            reach = int(pos[:n].max())
            tb.k_kv_move(kt, vt, [a for a, _ in pairs], [b for _, b in pairs], c, tb.KV_Q4, B, reach)
            for j in range(2):
                host[j] = kv_q4.moved(host[j], pairs, TK, reach, [32, 4])
            order = list(range(n))
            for a, b in pairs:
                order[b] = a
            order = order[:len(keep)]
            live, pos, tokens, n = [live[i] for i in order], pos[order], tokens[order], len(keep)
            if not n:
                break
        last, parts = forward(tokens, n, 1, int(pos[:n].max()), torch.tensor(pos[:n], dtype=torch.int32, device=DEV))
        follow(parts, n, 1, pos)
        pos = pos + 1
        if step % 2:                                       # a place that lags behind the others from here on
            pos[0] -= 1
    assert step == 11 or not live
