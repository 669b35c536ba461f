"""Sampling on the GPU against plain 64-bit arithmetic, row by row: every filter, equal logits, settings and random numbers at their ends, rows of one CTA and of several.

A weight is off by half a unit of 2^-44 at most (2^-45 of the largest) and by a few of the last bits of its exponential, so a sum over V tokens is off by V * 2^-45: 4e-9
at 128256 tokens and 1.5e-8 at the largest vocabulary, of a sum of 1 at least.  A token may differ from the oracle's only where a border of the cut or the draw lies so near, which for
the seeds here none does, or where numbers are equal by construction, which both sides hold exactly."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import sample  # noqa: E402
from paper_2609_06172_b200 import binding as tb  # noqa: E402

DEV = "cuda:0"


def run(logits, u, **settings):
    B, V = logits.shape
    dev = {n: torch.from_numpy(np.ascontiguousarray(np.broadcast_to(np.asarray(s, np.int32 if n == "top_k" else np.float32), (B,)))).to(DEV) for n, s in settings.items()}
    out = torch.full((B + 1,), -7, dtype=torch.int32, device=DEV)
    x = torch.from_numpy(np.ascontiguousarray(logits, np.float32)).to(DEV)
    tb.k_sample(x, torch.from_numpy(np.asarray(u, np.float32)).to(DEV), out, B, V, **dev)
    torch.cuda.synchronize()
    assert int(out[B]) == -7
    return out.cpu().numpy()[:B]


def check(logits, u, **settings):
    logits, u = np.asarray(logits, np.float32), np.asarray(u, np.float32)
    got = run(logits, u, **settings)
    each = {n: np.broadcast_to(np.asarray(s, np.int32 if n == "top_k" else np.float32), (len(u),)) for n, s in settings.items()}
    want = [sample.sample(logits[b], float(u[b]), **{n: (int if n == "top_k" else float)(s[b]) for n, s in each.items()}) for b in range(len(u))]
    assert list(got) == want, [(b, g, w) for b, (g, w) in enumerate(zip(got, want)) if g != w][:5]


SETTINGS = [dict(), dict(temperature=0.7), dict(top_k=5), dict(top_k=50, temperature=1.5), dict(top_p=0.9), dict(top_p=0.3, temperature=2.0), dict(min_p=0.05),
            dict(top_k=40, top_p=0.8), dict(temperature=0.8, top_k=100, top_p=0.95, min_p=0.02), dict(top_p=0.999, min_p=0.001), dict(top_k=1), dict(temperature=0.0)]


@pytest.mark.parametrize("V", [1, 2, 31, 512, 513, 4096, 4097, 32000, 50257, 128256])
@pytest.mark.parametrize("settings", SETTINGS, ids=str)
def test_filters(V, settings):
    rng = np.random.default_rng(V)
    B = 9 if V < 10000 else 5
    check(rng.standard_normal((B, V)) * np.array([0.1, 1, 2, 3, 6, 2, 2, 2, 2])[:B, None], rng.random(B), **settings)


@pytest.mark.parametrize("B", [1, 2, 37, 75, 150, 400])
def test_rows_with_settings_of_their_own(B):
    rng = np.random.default_rng(B)
    V = 9001
    check(rng.standard_normal((B, V)) * 2.5, rng.random(B), temperature=rng.choice([0.0, 0.5, 1.0, 1.7], B), top_k=rng.choice([0, 1, 20, 5000, V], B), top_p=rng.choice([0.0, 0.5, 0.95, 1.0], B),
          min_p=rng.choice([0.0, 0.1, 1.0], B))


@pytest.mark.parametrize("V", [600, 20000])
@pytest.mark.parametrize("settings", SETTINGS, ids=str)
def test_equal_logits(V, settings):
    """Logits on a grid: a cut falls among many that are equal, and the lower indices stay; all equal; two values."""
    rng = np.random.default_rng(V + 1)
    x = np.round(rng.standard_normal((6, V)) * 4) / 2
    x[1] = 3.25
    x[2] = np.where(np.arange(V) % 2, 1.0, 0.0)
    x[3] = -0.0
    x[3, ::3] = 0.0                                        # zeros of either sign are equal
    x[4] = np.round(x[4] * 8) / 16
    check(x, rng.random(6), **settings)


@pytest.mark.parametrize("top_k", [2, 3, 999, 1000, 1001, 19999, 20000, 2147483647, -1, -2147483648])
def test_top_k_at_its_ends(top_k):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 20000))
    x[1] = 0
    x[2, :1000] = 5                                        # a thousand equal ones before all others
    check(x, [0.0, 0.5, 0.99999994, 0.3], top_k=top_k)
    check(x, [0.9, 0.1, 0.7, 0.99999994], top_k=top_k, top_p=0.7)


@pytest.mark.parametrize("top_p", [0.0, -1.0, 1e-30, 1e-6, 0.5, 0.99999994, 1.0, 2.0, float("nan")])
def test_top_p_at_its_ends(top_p):
    rng = np.random.default_rng(6)
    x = rng.standard_normal((4, 5000)) * 3
    x[1] = 0                                               # the sum of the first so many is p by construction
    p = 1.0 if top_p != top_p else top_p
    got = run(x, [0.0, 0.5, 0.99999994, 0.3], top_p=top_p)
    assert list(got) == [sample.sample(x[b].astype(np.float32), u, top_p=float(np.float32(p))) for b, u in enumerate(np.float32([0.0, 0.5, 0.99999994, 0.3]).astype(float))]


@pytest.mark.parametrize("min_p", [0.0, -1.0, 1e-30, 0.5, 1.0, 1.5, float("nan")])
def test_min_p_at_its_ends(min_p):
    rng = np.random.default_rng(7)
    x = rng.standard_normal((3, 5000)) * 3
    x[1, [7, 99, 4000]] = 20                               # three that are as likely as the likeliest
    check(x, [0.0, 0.5, 0.99999994], min_p=0.0 if min_p != min_p else min_p)
    if min_p != min_p:
        assert list(run(x, [0.0, 0.5, 0.9], min_p=min_p)) == list(run(x, [0.0, 0.5, 0.9]))


@pytest.mark.parametrize("temperature", [1e-30, 1e-3, 1e3, 1e30, float("inf"), -1.0, float("nan")])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=30), dict(top_p=0.6), dict(top_k=300, top_p=0.6, min_p=0.5)], ids=str)
def test_temperatures_at_their_ends(temperature, settings):
    rng = np.random.default_rng(8)
    check(rng.standard_normal((3, 6000)) * 3, [0.0, 0.5, 0.99999994], temperature=temperature, **settings)


@pytest.mark.parametrize("V", [700, 9000])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=3), dict(top_p=0.6), dict(top_k=300, top_p=0.9), dict(temperature=0.0)], ids=str)
def test_tokens_that_are_masked_out(V, settings):
    """-inf and NaN are never drawn, a row of nothing else gives token 0; the type's lowest value is a logit like any other; infinities share all there is."""
    rng = np.random.default_rng(9)
    x = rng.standard_normal((9, V)).astype(np.float32) * 3
    x[0, rng.random(V) < 0.9] = -np.inf
    x[1, rng.random(V) < 0.5] = np.nan
    x[2] = -np.inf
    x[3] = np.nan
    x[4] = -np.inf
    x[4, V - 1] = -100.0
    x[5] = np.finfo(np.float32).min
    x[6] = np.finfo(np.float32).min
    x[6, 5:8] = 1.0
    x[7, [3, 400, 600]] = np.inf
    x[8, :] = np.nan
    x[8, 17] = np.inf
    for u in (0.0, 0.4, 0.99999994):
        check(x, [u] * 9, **settings)


def test_random_numbers_beyond_their_ends():
    x = np.log(np.array([[0.25, 0.25, 0.25, 0.25]] * 5))
    assert list(run(x, [-1.0, np.nan, 1.0, np.inf, 0.5])) == [0, 0, 3, 3, 2]


def test_weights_are_drawn_as_often_as_they_weigh():
    """Evenly spaced random numbers over a few tokens: each is drawn as often as its share, to one."""
    p = np.array([0.5, 0.125, 0.25, 0.0625, 0.0625])
    n = 4096
    x = np.tile(np.log(p), (n, 1))
    got = np.bincount(run(x, (np.arange(n) + 0.5) / n), minlength=5)
    assert (np.abs(got - p * n) <= 1).all()
    got = np.bincount(run(x, (np.arange(n) + 0.5) / n, top_k=3), minlength=5)
    assert (np.abs(got - np.array([0.5, 0.125, 0.25, 0, 0]) / 0.875 * n) <= 1).all()


def test_rows_that_do_not_begin_on_16_bytes():
    rng = np.random.default_rng(10)
    V = 9003
    x, u = rng.standard_normal((4, V)).astype(np.float32), rng.random(4).astype(np.float32)
    flat = torch.zeros(4 * V + 3, device=DEV)
    flat[1:4 * V + 1] = torch.from_numpy(x.reshape(-1)).to(DEV)
    out = torch.empty(4, dtype=torch.int32, device=DEV)
    tb.k_sample(flat.data_ptr() + 4, torch.from_numpy(u).to(DEV), out, 4, V, None, None, torch.full((4,), 0.8, device=DEV), None)
    assert out.tolist() == [sample.sample(x[b], float(u[b]), top_p=float(np.float32(0.8))) for b in range(4)]


def test_largest_vocabulary():
    rng = np.random.default_rng(12)
    check(rng.standard_normal((2, tb.SAMPLE_MAX_V)) * 2, rng.random(2), top_p=[0.9, 1.0])


@pytest.mark.parametrize("V", [tb.SAMPLE_MAX_V, 511591, 511590])
@pytest.mark.parametrize("settings", [dict(), dict(top_p=0.99), dict(min_p=0.5), dict(top_k=520000), dict(top_k=2147483647, top_p=0.9999999)], ids=str)
def test_flat_rows_of_the_largest_vocabulary(V, settings):
    """Sums of weights beyond 2^62, up to 2^63: equal logits and infinite temperatures, random numbers up to 1 and above."""
    rng = np.random.default_rng(13)
    u = np.float32([0.0, 0.5, 0.9758, 0.98, 0.99, 0.9999, 0.99999994])
    equal = np.full((len(u), V), 1.25, np.float32)
    check(equal, u, **settings)
    x = rng.standard_normal((3, V)).astype(np.float32)
    check(x, [0.98, 0.99, 0.99999994], temperature=float("inf"), **settings)
    assert list(run(equal[:4], [1.0, 2.0, np.inf, np.nan], **settings)) == [sample.sample(equal[0], 1.0, **{n: float(np.float32(s)) if n != "top_k" else s for n, s in settings.items()})] * 3 + [0]


def test_a_flat_row_of_a_large_vocabulary_is_drawn_evenly():
    """Of the largest vocabulary at a high temperature, by evenly spaced random numbers."""
    rng = np.random.default_rng(14)
    x = rng.standard_normal(tb.SAMPLE_MAX_V).astype(np.float32)
    u = np.float32((np.arange(8) + 0.5) / 8)
    check(np.tile(x, (8, 1)), u, temperature=1e3)


@pytest.mark.parametrize("V", [9000, 128256, tb.SAMPLE_MAX_V])
@pytest.mark.parametrize("below", [31.1, 31.3, 33.5])
def test_a_tail_at_the_end_of_the_weights(V, below):
    """One token before all others, which round to one unit of 2^-44 or to nothing: by V * 2^-45 at most, less than any random number below 1 tells."""
    x = np.full((4, V), -below, np.float32)
    x[:, V // 3] = 0
    for settings in (dict(), dict(top_p=0.9999999)):
        check(x, [1e-7, 0.5, 0.9999, 0.99999994], **settings)
    assert list(run(x[:2], [0.0, 1.0])) == ([0, V - 1] if below < 31.2 else [V // 3] * 2)


@pytest.mark.parametrize("temperature", [1.0, 3e37, 1e38, 3.4e38, float("inf")])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=30), dict(top_k=1000), dict(top_k=5500), dict(top_p=0.6), dict(top_p=0.95), dict(top_k=5000, top_p=0.9), dict(min_p=0.01)], ids=str)
def test_logits_whose_difference_is_no_number_of_fp32(temperature, settings):
    """The largest and the lowest logits lie further apart than fp32 reaches, and are as likely where the temperature is high enough."""
    rng = np.random.default_rng(15)
    top = np.finfo(np.float32).max
    x = np.stack([rng.choice([top, -top, 0.0, 1e38, -2e38], 6000), rng.choice([top, -top], 6000), np.where(np.arange(6000) == 4321, top, -top), rng.uniform(-1, 1, 6000) * top])
    for u in (0.0, 0.3, 0.7, 0.99999994):
        check(x, [u] * 4, temperature=temperature, **settings)
