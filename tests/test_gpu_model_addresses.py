"""Attention and adapters over planes and rows that lie beyond 4 GiB of their base."""
import numpy as np
import pytest

from model_harness import Batch, Cache, Rows
from oracle import model as M
from paper_2601_21473_amd import binding as B
from paper_2601_21473_amd.memory import DeviceBuffer
from test_gpu_adapters import Adapters
from test_gpu_prefix_attention import attend, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert B.device_count() > 0, "GPU tests need a GPU"


def spread(rng, bufs, chunks, units, big, capacity):
    """Copies units of `chunks` bytes, as bufs hold them, into planes of `capacity` units of
    `big` bytes, at places in no order of which the last is one.  Returns planes, places."""
    place = rng.choice(capacity - 1, units, replace=False)
    place[rng.integers(units)] = capacity - 1
    planes = [DeviceBuffer(capacity * big) for _ in bufs]
    for plane, buf, chunk in zip(planes, bufs, chunks):
        held = buf.download(0, units * chunk).reshape(units, chunk)
        for u in range(units):
            plane.upload(held[u], int(place[u]) * big)
    return planes, place


@pytest.mark.parametrize("kind,rows_kind", [(M.BF16, M.BF16), (M.E4M3, M.F16)])
@pytest.mark.parametrize("page,dim", [(16, 128), (4, 128), (16, 80)])
def test_attention(kind, rows_kind, page, dim):
    """Units beyond 4 GiB, read for few rows and for many, over a shared prefix too."""
    rng = np.random.default_rng(page + dim)
    lens = [40, 130, 90, 33]
    cache = Cache(rng, lens + [200], page=page, heads=2, dim=dim, kind=kind)
    big, capacity = 8 << 20, 600                     # 5 GB
    planes, place = spread(rng, cache.buf, [cache.chunk] * 2, cache.capacity, big, capacity)
    moved = place[cache.units].astype(np.int32)
    cache.d_units.upload(moved)
    cache.desc.capacity_units, cache.desc.k_unit_bytes, cache.desc.v_unit_bytes = capacity, big, big
    cache.desc.k, cache.desc.v = planes[0].ptr, planes[1].ptr
    batch = Batch([1, 60, 2, 1], range(4), lens, ([0, 2, 4], [4, 4], [200, 120]), spare=1)
    q = Rows(batch.n_rows, 6, dim, rows_kind, values=rng.standard_normal((batch.n_rows, 6, dim)))
    got, lse = attend(cache, batch, q, 3, rows_kind, scale=0.125)
    check(cache, batch, q, 3, rows_kind, got, lse, 0.125)
    for b in planes:
        b.free()


def test_attention_rows():
    """Rows of q and out 2 GiB apart, so that the last lie beyond 4 GiB."""
    rng = np.random.default_rng(1)
    lens, heads, dim, stride = [30, 70], 4, 64, 1 << 30
    cache = Cache(rng, lens, page=16, heads=2, dim=dim, kind=M.BF16)
    batch = Batch([1, 3], range(2), lens)
    near = Rows(4, heads, dim, M.BF16, values=rng.standard_normal((4, heads, dim)))
    want, _ = attend(cache, batch, near, 2, M.BF16, scale=0.2)
    q, out = (DeviceBuffer(2 * (3 * stride + heads * dim)) for _ in range(2))
    for t in range(4):
        q.upload(near.view(near.bytes)[t], 2 * t * stride)
    need = B.prefix_attention_workspace(cache.desc, batch.desc, heads)
    ws = DeviceBuffer(need)
    B.prefix_attention(cache.desc, batch.desc, q.ptr, out.ptr, type=M.BF16, n_q_heads=heads,
                       q_strides=(stride, dim), out_strides=(stride, dim), scale=0.2, workspace=ws.ptr,
                       workspace_bytes=need)
    B.null_stream_sync()
    for t in range(4):
        got = out.download(2 * t * stride, 2 * heads * dim).view(np.uint16).reshape(heads, dim)
        assert np.array_equal(got, want[t]), t
    for b in (q, out):
        b.free()


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("rows", [[1, 1, 0, 1], [2, 1, 3, 4], [40, 1, 30, 17]])
def test_adapters(kind, rows):
    """Units beyond 4 GiB, and rows of x, base and out of which the last lie beyond it.  Bounds as
    in test_gpu_adapters."""
    rng = np.random.default_rng(sum(rows))
    rank, n_in, n_out = 16, 264, 520
    ad = Adapters(rng, 4, rank, n_in, n_out, kind)
    units, big, capacity = len(ad.a), 64 << 20, 80   # 5 GB
    planes, place = spread(rng, ad.bufs[:2], ad.chunk, units, big, capacity)
    table = place[[ad.unit_of[a] for a in range(4)]].astype(np.int32)
    ad.bufs[2].upload(table)
    ad.desc.a, ad.desc.b, ad.desc.capacity_units = planes[0].ptr, planes[1].ptr, capacity
    ad.desc.a_unit_bytes = ad.desc.b_unit_bytes = big
    batch = Batch(rows, range(4), [0] * 4)
    n = batch.n_rows
    stride = ((5 << 30) // 2 // max(n - 1, 1) + 7) // 8 * 8
    x, y = M.to_bits(rng.standard_normal((n, n_in)), kind), M.to_bits(rng.standard_normal((n, n_out)), kind)
    d_x, d_y = (DeviceBuffer(2 * ((n - 1) * stride + m)) for m in (n_in, n_out))
    for t in range(n):
        d_x.upload(x[t], 2 * t * stride)
        d_y.upload(y[t], 2 * t * stride)
    need = B.adapter_add_workspace(ad.desc, n, 4)
    ws = DeviceBuffer(need)
    B.adapter_add(ad.desc, batch.desc, d_x.ptr, d_y.ptr, d_y.ptr, x_stride=stride, base_stride=stride,
                  out_stride=stride, workspace=ws.ptr, workspace_bytes=need)
    B.null_stream_sync()
    got = np.stack([d_y.download(2 * t * stride, 2 * n_out).view(np.uint16) for t in range(n)])
    u = M.HALF_STEP[kind]
    for r in range(4):
        at = slice(int(batch.row_off[r]), int(batch.row_off[r + 1]))
        am, bm = (M.from_bits(m[ad.unit_of[r]], kind) for m in (ad.a, ad.b))
        xv, yv = M.from_bits(x[at], kind), M.from_bits(y[at], kind)
        want, second, first = M.adapter(xv, am, bm, yv, 1.0)
        tol = u * np.abs(want) + (u * u + (2 * rank + 8) * 2.0 ** -24) * second + \
            (n_in + 40) * 2.0 ** -24 * first + 2.0 ** -23 * np.abs(yv)
        if kind == M.F16:
            top = np.abs(xv @ am.T).max(-1, initial=0)[:, None]
            tol = tol + 2.0 ** -39 * top * np.abs(bm).sum(1)[None] + 2.0 ** -25
        assert (np.abs(M.from_bits(got[at], kind) - want) <= tol).all(), r
    for b in planes + [d_x, d_y]:
        b.free()
