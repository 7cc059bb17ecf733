"""ss_adapter_add where a value or a size is at its edge, against the plain form in 64 bits."""
import numpy as np
import pytest

from model_harness import SENTINEL, Batch, Rows
from oracle import model as M
from paper_2601_21473_amd import binding as B
from paper_2601_21473_amd.memory import DeviceBuffer
from test_gpu_adapters import Adapters, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert B.device_count() > 0, "GPU tests need a GPU"


def fill(ad, a, b):
    """Every unit's matrices become a [rank, n_in] and b [n_out, rank]."""
    for i, (held, x) in enumerate(((ad.a, a), (ad.b, b))):
        held[:] = M.to_bits(x, ad.kind)
        raw = np.zeros((len(held), ad.chunk[i]), np.uint8)
        raw[:, :2 * x.size] = held.reshape(len(held), -1).view(np.uint8)
        ad.bufs[i].upload(raw)


@pytest.mark.parametrize("rows", [[1, 0, 1, 1], [2, 3], [20, 40, 1]])
@pytest.mark.parametrize("rank", [16, 40])
def test_fp16_sums_far_below_the_rows_largest(rows, rank):
    """A x has an element of 1,024 times the row, which B does not use, beside elements
    2^20 and more below it, which make the output.

    A row of A x is held in two fp16 parts under a power of two that brings its largest to
    2^14 at least.  A part's step below the normal range is 2^-24, so an element is off by
    2^-22 of itself (two roundings to half a step, 2^-11) or by 2^-25 of 2^-14 of the largest, 2^-39;
    B and the other terms as in test_gpu_adapters."""
    rng = np.random.default_rng(rank)
    n_in, n_out = 64, 264
    ad = Adapters(rng, 4, rank, n_in, n_out, M.F16)
    a, b = np.zeros((rank, n_in)), rng.uniform(1, 2, (n_out, rank))
    a[0, 0], b[:, 0] = 1024.0, 0.0
    a[1:, 1] = rng.uniform(1, 2, rank - 1) * 2.0 ** -10 * 2.0 ** -rng.integers(0, 4, rank - 1)
    fill(ad, a, b)
    batch = Batch(rows, range(len(rows)), [0] * len(rows))
    x = np.zeros((batch.n_rows, 1, n_in))
    x[:, 0, 0] = rng.choice([-1.0, 1.0, 2.0], batch.n_rows)
    x[:, 0, 1] = rng.uniform(0.5, 1, batch.n_rows)
    d_x = Rows(batch.n_rows, 1, n_in, M.F16, values=x)
    base = Rows(batch.n_rows, 1, n_out, M.F16, values=np.zeros((batch.n_rows, 1, n_out)))
    need = B.adapter_add_workspace(ad.desc, batch.n_rows, len(rows))
    ws = DeviceBuffer(need)
    B.adapter_add(ad.desc, batch.desc, d_x.ptr, base.ptr, base.ptr, x_stride=n_in, base_stride=n_out,
                  out_stride=n_out, workspace=ws.ptr, workspace_bytes=need)
    B.null_stream_sync()
    xv = d_x.before()[:, 0]
    am, bm = M.from_bits(ad.a[0], M.F16), M.from_bits(ad.b[0], M.F16)
    want, second, first = M.adapter(xv, am, bm, 0.0, 1.0)
    top = np.abs(xv @ am.T).max(-1)[:, None]
    tol = 2.0 ** -11 * np.abs(want) + (2.0 ** -22 + (2 * rank + 8) * 2.0 ** -24) * second + \
        (n_in + 40) * 2.0 ** -24 * first + 2.0 ** -39 * top * np.abs(bm).sum(1)[None] + 2.0 ** -25
    err = np.abs(base.values()[:, 0] - want)
    assert (err <= tol).all(), (err.max(), tol.min(), np.abs(want).min())


def test_more_workgroups_than_one_grid_dimension():
    """2^20 - 1 requests, nearly all of no rows, over a wide projection: 58 million
    workgroups of 256 threads, where a dimension of a grid ends at 2^32 threads.  Bounds
    as in test_gpu_adapters, without an fp16 part."""
    rng = np.random.default_rng(1)
    rank, n_in, n_out = 128, 8, 14336
    ad = Adapters(rng, 4, rank, n_in, n_out, M.BF16, away=(3,))
    rows = np.zeros((1 << 20) - 1, np.int64)
    used = [0, 5, 6, 1 << 19, len(rows) - 1]
    rows[used] = [1, 1, 2, 1, 3]
    agents = np.arange(len(rows)) % 3
    agents[5] = 3
    batch = Batch(rows, agents, np.zeros(len(rows)), spare=1)
    x = Rows(batch.n_rows, 1, n_in, M.BF16, values=rng.standard_normal((batch.n_rows, 1, n_in)))
    base = Rows(batch.n_rows, 1, n_out, M.BF16, values=rng.standard_normal((batch.n_rows, 1, n_out)))
    out = Rows(batch.n_rows, 1, n_out, M.BF16)
    need = B.adapter_add_workspace(ad.desc, batch.n_rows, len(rows))
    ws = DeviceBuffer(need)
    B.adapter_add(ad.desc, batch.desc, x.ptr, base.ptr, out.ptr, x_stride=n_in, base_stride=n_out,
                  out_stride=n_out, workspace=ws.ptr, workspace_bytes=need)
    B.null_stream_sync()
    got, clean = out.bits()
    assert clean
    xv, bv = x.before()[:, 0], base.before()[:, 0]
    for r in used:
        at = slice(int(batch.row_off[r]), int(batch.row_off[r + 1]))
        unit = ad.unit_of[agents[r]]
        if unit < 0:
            assert np.array_equal(got[at, 0], base.view(base.bytes)[at, 0]), r
            continue
        am, bm = M.from_bits(ad.a[unit], M.BF16), M.from_bits(ad.b[unit], M.BF16)
        want, second, first = M.adapter(xv[at], am, bm, bv[at], 1.0)
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -16 + (2 * rank + 8) * 2.0 ** -24) * second + \
            (n_in + 40) * 2.0 ** -24 * first + 2.0 ** -23 * np.abs(bv[at])
        assert (np.abs(M.from_bits(got[at, 0], M.BF16) - want) <= tol).all(), r
    assert (got[int(batch.row_off[-1]):] == SENTINEL * 0x101).all()


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("rank", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("rows", [[1] * 9, [0, 1, 5, 0, 0, 2, 0, 1, 0, 9, 0, 0, 0, 0, 0, 0, 0, 0],
                                  [1, 0, 1, 1, 2]])
def test_no_more_rows_than_requests(kind, rank, rows):
    """Decoding as a rule: outputs column by column, of requests of none to nine rows too,
    several with one adapter, one away, one that does not exist."""
    rng = np.random.default_rng(rank + len(rows))
    ad = Adapters(rng, 6, rank, 264, 1048, kind, away=(4,))
    agents = [0, 3, 3, 1, 4, 0, 5, 77, 2] * 2
    for in_place in (False, True):
        run(ad, Batch(rows, agents[:len(rows)], [0] * len(rows)), scales=rng.uniform(-2, 2, len(rows)),
            in_place=in_place, pad=0 if in_place else 8, seed=rank)


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("rank,n_out", [(8, 8200), (16, 4104), (32, 2568), (64, 1288), (128, 1032)])
def test_many_single_rows(kind, rank, n_out):
    """Requests enough that a wave takes two rounds of columns, the last of them partly."""
    rng = np.random.default_rng(n_out)
    ad = Adapters(rng, 30, rank, 64, n_out, kind, away=(7, 8))
    rows = np.ones(256, np.int64)
    rows[[3, 90]], rows[[4, 5]] = 2, 0
    run(ad, Batch(rows, rng.integers(0, 31, 256), [0] * 256), scales=rng.uniform(-2, 2, 256), seed=rank)


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("rank", [24, 32, 72, 128])
@pytest.mark.parametrize("n_in", [8, 1000])
def test_long_requests(kind, rank, n_in):
    """More than 16 rows a request as a rule: tiles of 32."""
    rng = np.random.default_rng(rank + n_in)
    ad = Adapters(rng, 4, rank, n_in, 776, kind, away=(2,))
    run(ad, Batch([40, 17, 3, 60, 0, 32], [0, 1, 2, 3, 1, 0], [0] * 6, spare=1),
        scales=rng.uniform(-2, 2, 6), in_place=rank == 32, seed=rank)


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("n,rows", [(20, 33), (60, 9)])
@pytest.mark.parametrize("rank", [16, 48])
def test_several_rounds_of_columns(kind, n, rows, rank):
    """Tiles enough that a workgroup takes several rounds of 512 columns, the last partly."""
    rng = np.random.default_rng(n + rank)
    ad = Adapters(rng, 5, rank, 128, 8200, kind, away=(1,))
    run(ad, Batch([rows] * n, rng.integers(0, 5, n), [0] * n), scales=rng.uniform(-2, 2, n), seed=n)


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 2, 4], [30, 20, 1]])
def test_infinite_and_nan_elements(kind, rows):
    """What an infinity or NaN of x, A or B takes part in is infinite or NaN, and nothing
    else: a row of x, a column of B, and all outputs of one adapter for A."""
    rng = np.random.default_rng(9)
    ad = Adapters(rng, 3, 16, 64, 72, kind)
    ad.b[ad.unit_of[0], 5, 3] = M.to_bits([np.inf], kind)[0]
    ad.b[ad.unit_of[1], 70, 15] = M.to_bits([np.nan], kind)[0]
    ad.a[ad.unit_of[2], 7, 9] = M.to_bits([-np.inf], kind)[0]
    for i, m in enumerate((ad.a, ad.b)):
        raw = np.zeros((len(m), ad.chunk[i]), np.uint8)
        raw[:, :m[0].nbytes] = m.reshape(len(m), -1).view(np.uint8)
        ad.bufs[i].upload(raw)
    batch = Batch(rows, [0, 1, 2], [0] * 3)
    n = batch.n_rows
    xv = rng.standard_normal((n, 1, 64))
    if rows[0] > 1:
        xv[1, 0, 20] = np.inf
    x = Rows(n, 1, 64, kind, values=xv)
    out = Rows(n, 1, 72, kind, values=np.zeros((n, 1, 72)))
    need = B.adapter_add_workspace(ad.desc, n, 3)
    ws = DeviceBuffer(need)
    B.adapter_add(ad.desc, batch.desc, x.ptr, out.ptr, out.ptr, x_stride=64, base_stride=72, out_stride=72,
                  workspace=ws.ptr, workspace_bytes=need)
    B.null_stream_sync()
    got = np.isfinite(out.values()[:, 0])
    want = np.ones((n, 72), bool)
    want[:rows[0], 5] = False
    want[rows[0]:rows[0] + rows[1], 70] = False
    want[rows[0] + rows[1]:] = False
    if rows[0] > 1:
        want[1] = False
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
