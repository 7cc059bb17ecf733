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
