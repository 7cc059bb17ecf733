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
