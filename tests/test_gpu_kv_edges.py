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


@pytest.mark.parametrize("kind", [M.BF16, M.E4M3])
def test_two_rows_for_one_token(kind):
    """Agent 0 in three requests, two of which give it the same tokens: what those hold may be
    anything, the other tokens and every byte beside them are as the rows say."""
    rng = np.random.default_rng(2)
    cache = Cache(rng, [40, 20], page=16, heads=3, dim=64, kind=kind)
    batch = Batch([6, 9, 4, 2], [0, 1, 0, 0], [30, 20, 27, 40])
    new = [Rows(batch.n_rows, 3, 64, M.BF16, values=rng.standard_normal((batch.n_rows, 3, 64)))
           for _ in range(2)]
    before = [b.copy() for b in cache.bytes]
    B.kv_write(cache.desc, batch.desc, new[0].ptr, new[1].ptr, type=M.BF16, strides=new[0].strides)
    B.null_stream_sync()
    request, token = M.positions(batch.row_off, batch.lens)
    twice = sorted(set(range(24, 30)) & set(range(23, 27)))
    got = cache.download()
    for i in range(2):
        x = new[i].before()
        want = before[i].copy()
        for t in range(len(request)):
            u, slot = cache.place(int(batch.agents[request[t]]), int(token[t]))
            if kind == M.E4M3:
                s = M.e4m3_scale(x[t])
                cache.scale_view(want)[u, :, slot] = s
                cache.body(want)[u, :, slot] = M.e4m3_encode(x[t].astype(np.float32) / s[:, None])
            else:
                cache.body(want)[u, :, slot] = new[i].view(new[i].bytes)[t]
        for p in (got[i], want):
            for token_twice in twice:
                u, slot = cache.place(0, token_twice)
                cache.body(p)[u, :, slot] = 0
                if kind == M.E4M3:
                    cache.scale_view(p)[u, :, slot] = 0
        assert np.array_equal(got[i], want)
