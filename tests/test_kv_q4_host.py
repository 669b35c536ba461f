"""What the calls on 4-bit tiles, the moves and the sampling refuse, and the sizes they tell: decided on the host, without a GPU.  The oracle's own rounding against
closed forms."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv_q4, sample
from paper_2609_06172_b200 import binding as tb

A = 4096                                                   # an address that nothing reads: every call here returns before it would


@pytest.fixture(params=["extension", "ctypes"], autouse=True)
def way(request, monkeypatch):
    """Every call both ways: through the extension, which serves exact lists and integers, and through ctypes."""
    tb.lib()
    if request.param == "ctypes":
        monkeypatch.setattr(tb, "_fast", tb._General())


def cfg(**over):
    c = dict(L=1, d=256, Hq=8, Hkv=2, Dh=64, F=1, V=1, E=0, topk=0, B=4, max_len=256, TK=32, rope_base=10000.0, eps=1e-5)
    return tb.ModelCfg(**{**c, **over})


def refused(code, f, *args, **kw):
    with pytest.raises(tb.TgpError) as e:
        f(*args, **kw)
    assert e.value.code == code, e.value


def attn(c=None, tiles=8, B=4, S=1, pos0=10, k_exp=0, v_exp=0, pos=None, q=A, o=A, scratch=A, kt=None, vt=None):
    tb.k_attn_q4(q, [A] * tiles if kt is None else kt, [A] * tiles if vt is None else vt, o, c or cfg(), B, S, pos0, k_exp, v_exp, pos, scratch)


def append(c=None, tiles=8, B=4, S=1, pos0=10, k_exp=0, v_exp=0, pos=None, q=A, cos=A, kt=None):
    tb.k_rope_kv_q4(q, A, A, A, [A] * tiles if kt is None else kt, [A] * tiles, cos, A, c or cfg(), B, S, pos0, k_exp, v_exp, pos)


def unpack(c=None, tiles=8, B=4, S=1, pos0=10, k_exp=0, v_exp=0, pos=None, out=A, kt=None):
    tb.k_kv_unpack_q4([A] * tiles if kt is None else kt, [A] * tiles, out, A, c or cfg(), B, S, pos0, k_exp, v_exp, pos)


@pytest.mark.parametrize("call", [attn, append, unpack])
def test_calls_on_4_bit_tiles_refuse(call):
    for bad in (dict(Dh=32), dict(Dh=96), dict(Dh=256), dict(TK=8), dict(TK=24), dict(TK=0), dict(Hkv=0), dict(Hq=7), dict(Hq=0)):
        refused(tb.E_INVAL, call, cfg(**bad))
    refused(tb.E_INVAL, call, B=5)                         # more sequences than the tiles hold
    refused(tb.E_INVAL, call, pos0=256)                    # behind max_len
    refused(tb.E_INVAL, call, pos0=250, S=7)
    refused(tb.E_INVAL, call, tiles=1, pos0=32)            # behind the tiles
    refused(tb.E_INVAL, call, S=2, pos=A)                  # positions of their own are for single tokens
    refused(tb.E_INVAL, call, k_exp=33)
    refused(tb.E_INVAL, call, v_exp=-33)
    refused(tb.E_TOO_LARGE, call, tiles=65)
    refused(tb.E_INVAL, call, kt=[A + 8] + [A] * 7)        # a tile that does not begin on 16 bytes
    refused(tb.E_INVAL, call, kt=[None] + [A] * 7)         # a tile that the call needs
    for pos0, S in ((4294967295, 1), (1, 4294967295)):
        refused(tb.E_INVAL, call, cfg(max_len=4294967295), pos0=pos0, S=S)
    call(B=0), call(S=0, pos0=0)                           # nothing to do


def test_batches_beyond_a_grid_are_refused():
    refused(tb.E_TOO_LARGE, unpack, cfg(B=32768), B=32768)              # 65536 pages
    refused(tb.E_TOO_LARGE, attn, cfg(B=65536), B=65536)
    refused(tb.E_TOO_LARGE, attn, cfg(B=65536), B=65536, S=40)
    refused(tb.E_TOO_LARGE, append, cfg(B=1 << 30), B=1 << 30, S=2)


def test_missing_and_misaligned_arguments():
    for kw in (dict(q=None), dict(o=None), dict(scratch=None), dict(q=A + 2), dict(o=A + 8), dict(scratch=A + 4)):
        refused(tb.E_INVAL, attn, **kw)
    for kw in (dict(q=None), dict(q=A + 4), dict(cos=None), dict(cos=A + 8)):
        refused(tb.E_INVAL, append, **kw)
    for kw in (dict(out=None), dict(out=A + 2)):
        refused(tb.E_INVAL, unpack, **kw)


def test_tiles_without_a_position_of_the_call_may_be_missing():
    tiles = [None, A] + [None] * 6
    refused(tb.E_INVAL, append, kt=[A, None] + [A] * 6, pos0=32)
    append(kt=tiles, pos0=32, B=0)
    refused(tb.E_INVAL, append, kt=tiles, pos0=32, pos=A)  # any of the earlier positions may be asked for
    refused(tb.E_INVAL, attn, kt=tiles, pos0=32)


def test_bytes_of_tiles_and_scratch():
    assert tb.k_kv_q4_tile_bytes(cfg()) == 4 * 2 * 32 * (32 + 4)
    assert tb.k_kv_q4_tile_bytes(cfg(Dh=128, TK=256, Hkv=8, B=61)) == 61 * 8 * 256 * 72
    refused(tb.E_INVAL, tb.k_kv_q4_tile_bytes, cfg(Dh=80))
    for q_len in (0, 257):
        refused(tb.E_INVAL, tb.k_attn_q4_scratch_bytes, cfg(), q_len)
    refused(tb.E_INVAL, tb.k_attn_q4_scratch_bytes, cfg(B=0), 1)
    # a batch that has shrunk needs no more than the whole one
    for B in (1, 3, 64, 1000):
        sizes = [tb.k_attn_q4_scratch_bytes(cfg(B=b, max_len=16384, TK=256), 1) for b in range(1, B + 1)]
        assert sizes == sorted(sizes)
    # from 32 queries on the keys and values fit as bf16, a whole number of 64 positions of them
    for max_len in (65536, 65500):
        assert tb.k_attn_q4_scratch_bytes(cfg(max_len=max_len, TK=1024), 32) == 2 * 4 * 2 * 65536 * 64 * 2
    assert tb.k_attn_q4_scratch_bytes(cfg(max_len=65536, TK=1024), 31) < 1 << 24


def test_scratch_for_an_unpacked_cache_is_limited():
    """4 GiB for as many sequences as fit, one sequence's where that is more; what fits entirely takes what it takes."""
    long = dict(Hq=64, Hkv=8, Dh=128, max_len=131072, TK=2048)
    one = 2 * 8 * 131072 * 128 * 2                         # 512 MiB
    for B, sequences in ((1, 1), (7, 7), (8, 8), (9, 8), (64, 8), (1000, 8)):
        assert tb.k_attn_q4_scratch_bytes(cfg(**long, B=B), 32) == tb.k_attn_q4_scratch_bytes(cfg(**long, B=B), 131072) == sequences * one
    for B in (1, 5):
        assert tb.k_attn_q4_scratch_bytes(cfg(Hq=64, Hkv=32, Dh=128, max_len=1 << 20, TK=1 << 14, B=B), 64) == 2 * 32 * (1 << 20) * 128 * 2


def move(src, dst, c=None, form=tb.KV_Q4, B=4, length=40, tiles=2, kt=None):
    tb.k_kv_move([A] * tiles if kt is None else kt, [A] * tiles, src, dst, c or cfg(), form, B, length)


def test_moves_refuse():
    refused(tb.E_INVAL, move, [0], [4])                    # no such place
    refused(tb.E_INVAL, move, [4], [0])
    refused(tb.E_INVAL, move, [-2], [0])
    refused(tb.E_INVAL, move, [0], [-1])
    refused(tb.E_INVAL, move, [0, 1], [2, 2])              # one destination twice
    refused(tb.E_INVAL, move, [2, 1], [2, 2])              # ... also where it is its own source
    refused(tb.E_INVAL, move, [0] * 5, [0, 1, 2, 3, 3])    # more pairs than places
    refused(tb.E_INVAL, move, [0], [1], B=5)
    refused(tb.E_INVAL, move, [0], [1], form=2)
    refused(tb.E_INVAL, move, [0], [1], length=65)         # behind the tiles
    refused(tb.E_INVAL, move, [0], [1], length=257, tiles=16)
    refused(tb.E_INVAL, move, [0], [1], c=cfg(Dh=80))      # 4 bits hold 64 or 128 dimensions
    refused(tb.E_INVAL, move, [0], [1], c=cfg(Dh=12), form=tb.KV_BF16)
    refused(tb.E_INVAL, move, [0], [1], c=cfg(TK=20))
    refused(tb.E_INVAL, move, [0], [1], kt=[A, None])
    refused(tb.E_INVAL, move, [0], [1], kt=[A, A + 4])
    refused(tb.E_TOO_LARGE, move, [0], [1], tiles=65)
    refused(tb.E_TOO_LARGE, move, [0], [1], c=cfg(B=40000), B=40000)
    with pytest.raises(ValueError):
        move([0, 1], [2])
    move([], [])                                           # nothing to do
    move([1], [1])
    move([0], [1], length=0, kt=[None, None])


def test_sampling_refuses():
    for args in ((None, A, A, 1, 10), (A, None, A, 1, 10), (A, A, None, 1, 10), (A, A, A, 1, 0)):
        refused(tb.E_INVAL, tb.k_sample, *args)
    refused(tb.E_TOO_LARGE, tb.k_sample, A, A, A, 1, tb.SAMPLE_MAX_V + 1)
    tb.k_sample(A, A, A, 0, 10)


def test_other_kinds_of_arguments_are_the_same_call():
    """Tuples, arrays and generators of numbers take the general path, with the same checks."""
    c = cfg()
    for src, dst in (((0, 1), (2, 2)), (np.array([0, 1]), np.array([2, 2])), ([0, 1], np.array([2, 2]))):
        refused(tb.E_INVAL, tb.k_kv_move, (A, A), [A, A], src, dst, c, tb.KV_Q4, 4, 40)
    refused(tb.E_INVAL, tb.k_attn_q4, A, (A,) * 8, [A] * 8, A, c, 5, 1, 10, 0, 0, None, A)
    refused(tb.E_INVAL, tb.k_attn_q4, A, [A] * 8, [A] * 8, A, c, np.uint32(4), 1, 300, scratch=A)
    refused(tb.E_INVAL, tb.k_sample, A, A, A, np.int64(1), 0)
    with pytest.raises((TypeError, C.ArgumentError)):
        tb.k_attn_q4(A, [A] * 8, [A] * 8, A, c, 4, 1, 10, 0.5, 0, None, A)


def test_null_configurations():
    n, t = tb._U64(), (tb._P * 1)(A)
    l = tb.lib()
    assert l.tgp_k_kv_q4_tile_bytes(None, C.byref(n)) == tb.E_INVAL and l.tgp_k_kv_q4_tile_bytes(C.byref(cfg()), None) == tb.E_INVAL
    assert l.tgp_k_attn_q4_scratch_bytes(None, 1, C.byref(n)) == tb.E_INVAL
    assert l.tgp_k_attn_q4(A, t, t, 1, A, None, 1, 1, 0, 0, 0, None, A, None) == tb.E_INVAL
    assert l.tgp_k_attn_q4(A, None, t, 1, A, C.byref(cfg()), 1, 1, 0, 0, 0, None, A, None) == tb.E_INVAL
    assert l.tgp_k_kv_move(t, None, 1, None, None, 0, C.byref(cfg()), 1, 1, 1, None) == tb.E_INVAL
    assert l.tgp_k_kv_move(t, t, 1, None, None, 1, C.byref(cfg()), 1, 1, 1, None) == tb.E_INVAL


# ---- the oracle against closed forms ----

def test_oracle_rounding():
    assert list(kv_q4.E4M3[[0, 1, 7, 8, 0x38, 0x7e]]) == [0, 2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 1.0, 448.0] and np.isnan(kv_q4.E4M3[[0x7f, 0xff]]).all()
    x = np.zeros((1, 16))
    x[0, :9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5]            # scale 1: every border goes to the even code
    codes, scales = kv_q4.quantise(x, 0)
    assert list(kv_q4.values(codes, scales, 0)[0, :9]) == [6, 0, 1, 1, 2, 2, 4, 4, -4] and scales[0, 0] == 0x38
    for exp in (-32, -5, 7, 32):                                        # a power of two goes with the exponent
        c2, s2 = kv_q4.quantise(x * 2.0 ** exp, exp)
        assert (c2 == codes).all() and (s2 == scales).all()
    big, s = kv_q4.quantise(np.full((1, 16), 1e6), 0)                   # beyond the largest
    assert kv_q4.values(big, s, 0)[0, 0] == 6 * 448
    tiny, s = kv_q4.quantise(np.full((1, 16), 6 * 2.0 ** -11), 0)       # a scale that rounds to 0
    assert s[0, 0] == 0 and not kv_q4.values(tiny, s, 0).any()
    bad, s = kv_q4.quantise(np.array([[1.0] * 15 + [np.inf] + [3.0] * 16]), 0)
    assert s[0, 0] == 127 and np.isnan(kv_q4.values(bad, s, 0)[0, :16]).all() and (kv_q4.values(bad, s, 0)[0, 16:] == 3).all()


def test_oracle_attention_of_equal_keys_is_the_mean():
    rng = np.random.default_rng(1)
    V = rng.standard_normal((2, 9, 64))
    o, mean, *_ = kv_q4.attention(rng.standard_normal((3, 4, 64)), np.ones((2, 9, 64)), V, 6)
    for t in range(3):
        assert np.allclose(o[t, 3], V[1, :7 + t].mean(0)) and np.allclose(mean[t, 0], np.abs(V[0, :7 + t]).mean(0))


def test_oracle_sampling():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    assert [sample.sample(x, u) for u in (0.0, 0.0999, 0.1001, 0.4999, 0.5001, 0.6999, 0.7001, 0.9999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [sample.sample(x, u, top_k=2) for u in (0.0, 0.57, 0.58)] == [1, 1, 3]
    assert [sample.sample(x, u, top_p=0.69) for u in (0.0, 0.57, 0.58)] == [1, 1, 3] and sample.sample(x, 0.99, top_p=0.39) == 1
    assert [sample.sample(x, u, min_p=0.6) for u in (0.0, 0.57, 0.58)] == [1, 1, 3]
    assert sample.sample(x, 0.99, temperature=0.0) == 1 and sample.sample([np.nan, -np.inf], 0.5) == 0
    assert [sample.sample([1.0, 1.0, 1.0], u, top_k=2) for u in (0.4, 0.99)] == [0, 1]
    assert sample.sample([np.inf, 0.0, np.inf], 0.7) == 2
