"""ss_kv_write and ss_kv_read at the edge of their sizes and rules."""
import numpy as np
import pytest

from model_harness import SENTINEL, Batch, Cache, Rows, up
from oracle import model as M
from paper_2601_21473_amd import binding as B
from paper_2601_21473_amd.memory import DeviceBuffer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert B.device_count() > 0, "GPU tests need a GPU"


@pytest.mark.parametrize("kind", [M.BF16, M.E4M3])
def test_more_workgroups_than_one_grid_dimension(kind):
    """2^28 + 100 rows of one agent: 2^24 and a few workgroups of 256 threads, where a
    dimension of a grid ends at 2^32 threads.  The first and the last page are resident."""
    n, page, dim = (1 << 28) + 100, 1024, 16
    size = 1 if kind == M.E4M3 else 2
    chunk = page * dim * size + (4 * page if size == 1 else 0)
    pages = -(-n // page)
    units = np.full(pages, -1, np.int32)
    units[0], units[-1] = 1, 0
    planes = [up(np.full(2 * chunk, SENTINEL, np.uint8)) for _ in range(2)]
    d_units, d_off = up(units), up(np.array([0, pages], np.uint64))
    desc = B.kv_cache(units=d_units.ptr, agent_off=d_off.ptr, n_agents=1, n_entries=pages,
                      capacity_units=2, k=planes[0].ptr, v=planes[1].ptr, k_unit_bytes=chunk,
                      v_unit_bytes=chunk, page_tokens=page, n_heads=1, head_dim=dim, type=kind,
                      token_bytes=dim * size, head_bytes=page * dim * size,
                      scale_off=page * dim if size == 1 else 0)
    d_row_off, d_agents, d_lens = up(np.array([0, n], np.uint32)), up(np.zeros(1, np.uint32)), \
        up(np.array([n], np.uint32))
    batch = B.batch(n_rows=n, n_requests=1, row_off=d_row_off.ptr, agents=d_agents.ptr, lens=d_lens.ptr)
    # every row is the same one: powers of two below 448, so that e4m3 holds them
    x = 448.0 * 2.0 ** -np.arange(16.0).reshape(1, 1, 16).clip(0, 8)
    new = [Rows(1, 1, dim, M.BF16, values=y) for y in (x, -x)]
    B.kv_write(desc, batch, new[0].ptr, new[1].ptr, type=M.BF16, strides=(0, 0))
    B.null_stream_sync()
    for plane, y in zip(planes, (x, -x)):
        raw = plane.download(0, 2 * chunk).reshape(2, chunk)
        last = n - (pages - 1) * page                    # tokens of the last page
        for u, count in ((1, page), (0, last)):
            body = raw[u, :page * dim * size].copy().view(np.uint8 if size == 1 else np.uint16)
            v = M.from_bits(body[:count * dim], kind).reshape(count, dim)
            assert (v == y[0]).all()
            assert (raw[u, count * dim * size:page * dim * size] == SENTINEL).all()
            if size == 1:
                scales = raw[u, page * dim:].copy().view(np.float32)
                assert (scales[:count] == 1).all()
    out = [DeviceBuffer(n * dim * 2) for _ in range(2)]
    B.kv_read(desc, batch, out[0].ptr, out[1].ptr, type=M.BF16, strides=(dim, dim))
    B.null_stream_sync()
    for o, y in zip(out, (x, -x)):
        want = M.to_bits(y, M.BF16).reshape(1, dim)
        for first, count, there in ((0, page, True), (page, 5, False), (n - last - 5, 5, False),
                                    (n - last, last, True)):
            got = o.download(first * dim * 2, count * dim * 2).view(np.uint16).reshape(count, dim)
            assert (got == (want if there else 0)).all(), (first, there)
    for b in out + planes:
        b.free()
