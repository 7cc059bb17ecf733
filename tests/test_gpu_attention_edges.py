"""ss_prefix_attention where a value, a length or an address is at its edge, against the
plain form in 64 bits."""
import numpy as np
import pytest

from model_harness import Batch, Cache, Rows
from oracle import model as M
from paper_2601_21473_amd import binding as B
from test_gpu_prefix_attention import KINDS, attend, expected, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert B.device_count() > 0, "GPU tests need a GPU"


def set_contents(cache, keys, values):
    """Agent 0's tokens become keys and values [tokens, heads, dim]."""
    for i, x in enumerate((keys, values)):
        bits = M.to_bits(x, cache.kind)
        for t in range(len(x)):
            u, slot = cache.place(0, t)
            cache.bits[i, u, :, slot] = bits[t]
        cache._fill(i)
        cache.buf[i].upload(cache.bytes[i])


@pytest.mark.parametrize("page", [16, 4])
@pytest.mark.parametrize("rows,per,tokens", [(1, 2, 20_000), (3, 20, 8_000), (40, 4, 8_000)])
@pytest.mark.parametrize("where", ["first", "last"])
def test_fp16_weights_far_below_the_largest(page, rows, per, tokens, where):
    """One token has the whole weight but for e^-17.4 (2^-25.1) of each other one, and a
    value of 0 where theirs is 1, so the output is what the small weights add up to.

    Weights are held in fp16, the row's largest as 2^6 or more, and are off by half a step
    below the normal range, 2^-25, which is 2^-31 of the largest: n of them by n 2^-31 of
    the largest value in all.  The rest of the bound is as in test_gpu_prefix_attention."""
    rng = np.random.default_rng(tokens)
    cache = Cache(rng, [tokens], page=page, heads=1, dim=64, kind=M.F16)
    k, v = np.zeros((tokens, 1, 64)), np.ones((tokens, 1, 64))
    big = 0 if where == "first" else tokens - rows
    k[big, 0, 0], v[big] = 17.4, 0.0
    set_contents(cache, k, v)
    batch = Batch([rows], [0], [tokens])
    x = np.zeros((rows, per, 64))
    x[:, :, 0] = 1.0
    q = Rows(rows, per, 64, M.F16, values=x)
    got, lse = attend(cache, batch, q, per, M.F16, scale=1.0)
    (o, l, mag, _, size), count = expected(cache, batch, q.before(), per, 1.0)
    o, mag, l, size = o[:, 0], mag[:, 0], l[:, 0], size[:, 0]
    e = 68 * 2.0 ** -24 * size + 2.0 ** -21
    terms = (count[:, None] + 64) * 2.0 ** -24
    tol = (2.0 ** -11 + 4 * e + terms)[..., None] * mag + count[:, None, None] * 2.0 ** -31 + \
        2.0 ** -11 * np.abs(o) + 2.0 ** -25
    assert (np.abs(M.from_bits(got, M.F16) - o) <= tol).all(), (M.from_bits(got, M.F16)[0, 0, 0], o[0, 0, 0])
    assert (np.abs(lse - l) <= 2 * e + terms + 2.0 ** -22 * np.abs(l)).all()


@pytest.mark.parametrize("scale", [40.0, -40.0])
def test_fp16_weights_of_large_scores(scale):
    """Scores of several thousand: the reference moves far, weights stay within the type."""
    rng = np.random.default_rng(3)
    cache = Cache(rng, [300, 100], page=16, heads=2, dim=64, kind=M.F16, spread=2.0)
    run(cache, Batch([1, 30], [0, 1], [300, 100]), 2, M.F16, scale=scale, size=2.0)


@pytest.mark.parametrize("kind,rows_kind", KINDS)
@pytest.mark.parametrize("rows,lens,per", [
    ([3, 2, 5, 1], [1, 0, 7, 1], 2), ([30, 12, 3], [5, 12, 0], 4), ([90, 70], [3, 200], 1), ([6], [2], 2)])
@pytest.mark.parametrize("prefix", [1, 64, 150])
def test_rows_before_their_agents_first_token(kind, rows_kind, rows, lens, per, prefix):
    """More rows than tokens: the early ones see the prefix alone, all of it, in shared tiles
    of a group and in requests that read the prefix for themselves."""
    rng = np.random.default_rng(prefix)
    n = len(rows)
    cache = Cache(rng, lens + [prefix], page=16, heads=2, dim=64, kind=kind)
    run(cache, Batch(rows, range(n), lens, ([0, n], [n], [prefix]), spare=1), per, rows_kind)


@pytest.mark.parametrize("kind,rows_kind", KINDS)
@pytest.mark.parametrize("rows,per", [(1, 2), (30, 4)])
@pytest.mark.parametrize("shared", [False, True])
def test_scores_far_from_zero(kind, rows_kind, rows, per, shared):
    """Scores of 2^28 (fp16) and 2^40 (bf16), finite in 32 bits and further apart than any
    exponent reaches, but for two tokens whose scores are equal: the output is the mean of
    their values (weights 1 and 1, the sum 2), off by its own rounding and that of a sum of two,
    and the log-sum their score and ln 2, off by its rounding and the score's, 2^-22 of it.
    With e4m3 the weights are multiplied with the values' scales before they are rounded, so 1
    becomes a number of any bits and is off by half a step of bf16, 2^-8 of it, or of two
    parts, 2^-16."""
    rng = np.random.default_rng(rows)
    size = 2.0 ** (14 if rows_kind == M.F16 else 20)
    tokens, dim = 700, 64
    cache = Cache(rng, [tokens, tokens], page=16, heads=1, dim=dim, kind=kind)
    k = np.zeros((tokens, 1, dim))
    k[:, 0, 0] = -size * rng.uniform(0, 1, tokens)
    k[[3, 500], 0, 0] = size
    v = rng.standard_normal((tokens, 1, dim))
    held = [M.stored(M.from_bits(M.to_bits(x, rows_kind), rows_kind), kind) for x in (k, v)]
    new = [Rows(2 * tokens, 1, dim, rows_kind, values=np.concatenate([x, x])) for x in (k, v)]
    both = Batch([tokens] * 2, [0, 1], [tokens] * 2)
    B.kv_write(cache.desc, both.desc, new[0].ptr, new[1].ptr, type=rows_kind, strides=new[0].strides)
    n = 3 if shared else 1
    # alone: rows at the end of agent 0's tokens; shared: agent 0 is the prefix of requests
    # whose agents do not exist
    batch = Batch([rows] * n, [9] * n, [rows] * n, ([0, n], [0], [tokens])) if shared else \
        Batch([rows], [0], [tokens])
    x = np.zeros((n * rows, per, dim))
    x[:, :, 0] = size * rng.uniform(0.5, 1, (n * rows, per))
    q = Rows(n * rows, per, dim, rows_kind, values=x)
    got, lse = attend(cache, batch, q, per, rows_kind, scale=1.0)
    want = held[1][[3, 500], 0].mean(0)
    mag = np.abs(held[1][[3, 500], 0]).mean(0)
    err = np.abs(M.from_bits(got, rows_kind) - want)
    rounded = 0 if kind != M.E4M3 else 2.0 ** (-16 if rows_kind == M.F16 else -8)
    assert (err <= M.HALF_STEP[rows_kind] * np.abs(want) + (2.0 ** -22 + rounded) * mag + 2.0 ** -25).all()
    score = q.before()[:, :, 0] * held[0][3, 0, 0] + np.log(2)
    assert (np.abs(lse - score) <= 2.0 ** -22 * np.abs(score)).all()


@pytest.mark.parametrize("kind,rows_kind", KINDS)
@pytest.mark.parametrize("scale", [0.5, -8.0, 100.0, 1e6])
def test_scores_from_near_to_far(kind, rows_kind, scale):
    """Rows whose scores pass 2^12 beside rows whose scores do not, in the same tiles.

    The bound of test_gpu_prefix_attention, and what it leaves out: exponentials end at
    2^-126, so each of n weights, 1 for the largest, can be off by that, and by as much again
    when it is multiplied with a value's scale and rounded, before a code of up to 448:
    n 2^-117 (1 + max|v|) in all, where the largest weights meet values of 0."""
    rng = np.random.default_rng(11)
    lens = [200, 90, 333]
    cache = Cache(rng, lens + [150], page=16, heads=2, dim=64, kind=kind, spread=2.0)
    batch = Batch([1, 40, 3], range(3), lens, ([0, 3], [3], [150]))
    n = batch.n_rows
    x = rng.standard_normal((n, 6, 64)) * 2.0 ** rng.integers(-12, 4, (n, 6, 1))
    q = Rows(n, 6, 64, rows_kind, values=x)
    got, lse = attend(cache, batch, q, 3, rows_kind, scale=scale)
    (o, l, mag, big, size), count = expected(cache, batch, q.before(), 3, scale)
    o, mag, big = (y.reshape(n, 6, 64) for y in (o, mag, big))
    l, size = l.reshape(n, 6), size.reshape(n, 6)
    e = 68 * 2.0 ** -24 * size + 2.0 ** -21
    terms = (count[:, None] + 64) * 2.0 ** -24
    stored = M.BF16 if kind == M.E4M3 else kind
    u16 = M.HALF_STEP[stored] ** (2 if kind == M.E4M3 and rows_kind == M.F16 else 1)
    tol = (u16 + 4 * e + terms)[..., None] * mag + M.HALF_STEP[rows_kind] * np.abs(o) + \
        count[:, None, None] * 2.0 ** -117 * (1 + big)
    if stored == M.F16:
        tol = tol + count[:, None, None] * 2.0 ** -31 * big
    if rows_kind == M.F16:
        tol = tol + 2.0 ** -25
    value = M.from_bits(got, rows_kind)
    assert np.isfinite(value).all() and np.isfinite(lse).all()
    assert (np.abs(value - o) <= tol).all(), np.argwhere(np.abs(value - o) > tol)[:4]
    assert (np.abs(lse - l) <= 2 * e + terms + 2.0 ** -22 * np.abs(l)).all()
