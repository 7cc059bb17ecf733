"""The operators over resident units at the ends of what their arguments may be: most heads,
most query heads of a head, most requests and groups, long rows of an adapter."""
import numpy as np
import pytest

from model_harness import SENTINEL, Batch, Cache, Rows
from oracle import model as M
from paper_2601_21473_amd import binding as B
from test_gpu_adapters import Adapters
from test_gpu_adapters import run as run_adapters
from test_gpu_prefix_attention import KINDS, run

pytestmark = pytest.mark.gpu
MOST = (1 << 20) - 1


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert B.device_count() > 0, "GPU tests need a GPU"


@pytest.mark.parametrize("kind,rows_kind", KINDS)
@pytest.mark.parametrize("order", ["head", "token"])
def test_most_heads(kind, rows_kind, order):
    rng = np.random.default_rng(1)
    cache = Cache(rng, [5, 40], page=4, heads=1024, dim=16, kind=kind, order=order)
    run(cache, Batch([1, 3], [0, 1], [5, 40]), 1, rows_kind)
    cache = Cache(rng, [5, 9], page=4, heads=1024, dim=16, kind=kind, order=order)
    batch = Batch([1, 3], [0, 1], [5, 9])
    new = [Rows(4, 1024, 16, rows_kind, values=rng.standard_normal((4, 1024, 16))) for _ in range(2)]
    back = [Rows(4, 1024, 16, rows_kind) for _ in range(2)]
    B.kv_write(cache.desc, batch.desc, new[0].ptr, new[1].ptr, type=rows_kind, strides=new[0].strides)
    B.kv_read(cache.desc, batch.desc, back[0].ptr, back[1].ptr, type=rows_kind, strides=back[0].strides)
    B.null_stream_sync()
    for a, b in zip(new, back):
        want = M.stored(a.before(), kind)
        tol = 0 if kind != M.E4M3 else np.abs(want) * (M.HALF_STEP[rows_kind] + 2.0 ** -24) + 2.0 ** -25
        assert (np.abs(b.values() - want) <= tol).all()


@pytest.mark.parametrize("per", [300, 65536])
def test_most_query_heads(per):
    rng = np.random.default_rng(2)
    cache = Cache(rng, [70, 3, 100], page=16, heads=1, dim=16, kind=M.BF16)
    run(cache, Batch([1, 2], [0, 1], [70, 3], ([0, 2], [2], [100])), per, M.BF16)


def sparse(rng, n):
    rows = np.zeros(n, np.int64)
    used = np.unique(np.concatenate([[0, 1, n - 1], rng.integers(0, n, 20)]))
    rows[used] = rng.integers(1, 4, len(used))
    return rows, used


def test_most_requests_and_groups():
    """Nearly all requests have no rows and nearly all groups no requests."""
    rng = np.random.default_rng(3)
    rows, used = sparse(rng, MOST)
    lens = rng.integers(3, 60, 40)
    agents = rng.integers(0, 40, MOST)
    cache = Cache(rng, lens, page=16, heads=1, dim=16, kind=M.BF16)
    off = np.zeros(MOST + 1, np.int64)
    ends = np.sort(rng.choice(MOST, 30, replace=False))
    for i, e in enumerate(ends):
        off[e:] = (i + 1) * (MOST // 30)
    off[-1] = MOST
    prefix = rng.integers(0, 40, MOST)
    batch = Batch(rows, agents, lens[agents], (off, prefix, lens[prefix]), spare=2)
    # the group of a request, without a search through a million groups for each
    begin, end = off[:-1], off[1:]
    filled = np.flatnonzero(end > begin)
    by_request = {}
    for g in filled:
        for r in used[(used >= begin[g]) & (used < end[g])]:
            by_request[int(r)] = (int(prefix[g]), int(lens[prefix[g]]))
    batch.prefix_of = lambda r: by_request.get(int(r))
    run(cache, batch, 2, M.BF16)


@pytest.mark.parametrize("kind", [M.BF16, M.E4M3])
def test_tokens_of_most_requests(kind):
    rng = np.random.default_rng(4)
    rows, used = sparse(rng, MOST)
    lens = rng.integers(3, 60, 40)
    # every request that has rows has an agent of its own
    agents = np.full(MOST, 39)
    agents[used] = np.arange(len(used))
    cache = Cache(rng, lens, page=16, heads=2, dim=64, kind=kind)
    batch = Batch(rows, agents, lens[agents], spare=1)
    new = [Rows(batch.n_rows, 2, 64, M.BF16, values=rng.standard_normal((batch.n_rows, 2, 64)))
           for _ in range(2)]
    back = [Rows(batch.n_rows, 2, 64, M.BF16) for _ in range(2)]
    B.kv_write(cache.desc, batch.desc, new[0].ptr, new[1].ptr, type=M.BF16, strides=new[0].strides)
    B.kv_read(cache.desc, batch.desc, back[0].ptr, back[1].ptr, type=M.BF16, strides=back[0].strides)
    B.null_stream_sync()
    n = int(batch.row_off[-1])
    for a, b in zip(new, back):
        want = M.stored(a.before(), kind)[:n]
        got, clean = b.bits()
        tol = 0 if kind != M.E4M3 else np.abs(want) * (2.0 ** -8 + 2.0 ** -24)
        assert clean and (np.abs(M.from_bits(got[:n], M.BF16) - want) <= tol).all()
        assert (got[n:] == SENTINEL * 0x101).all()


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("rows", [[1, 1], [3, 20], [40]])
@pytest.mark.parametrize("n_in,n_out", [((1 << 18) + 8, 8), (8, (1 << 18) + 8)])
def test_long_rows_of_adapters(kind, rows, n_in, n_out):
    rng = np.random.default_rng(5)
    ad = Adapters(rng, 2, 8, n_in, n_out, kind)
    run_adapters(ad, Batch(rows, [1, 0][:len(rows)], [0] * len(rows)))
