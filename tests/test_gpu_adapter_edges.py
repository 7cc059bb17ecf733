"""ss_adapter_add where a value or a size is at its edge, against the plain form in 64 bits."""
import numpy as np
import pytest

from model_harness import SENTINEL, Batch, Rows
from oracle import model as M
from paper_2601_21473_amd import binding as B
from paper_2601_21473_amd.memory import DeviceBuffer
from test_gpu_adapters import Adapters

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
