"""ss_adapter_add against the plain form in 64 bits.

Bound per output: the first sum has n_in exact products in 32 bits, so it is off by
(n_in / 32 + 40) 2^-24 sum|A||x| at most where lanes and pieces add up in parallel
chains, taken as (n_in + 40) 2^-24; its two 16-bit parts keep it to u^2 (u half a
step of the type; fp16 parts below the type's normal range by 2^-25 of twice the
row's largest, under the row's power of two); the second sum of 2 rank products
adds (2 rank + 8) 2^-24; then the output's own rounding."""
import numpy as np
import pytest

from model_harness import SENTINEL, Batch, Rows, up
from oracle import model as M
from paper_2601_21473_amd import binding as B
from paper_2601_21473_amd.memory import DeviceBuffer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert B.device_count() > 0, "GPU tests need a GPU"


class Adapters:
    """Agents of `per` units each, of which unit `unit` holds this projection."""

    def __init__(self, rng, n, rank, n_in, n_out, kind, per=1, unit=0, away=(), size=1.0):
        self.rank, self.n_in, self.n_out, self.kind = rank, n_in, n_out, kind
        cap = n * per + 2
        self.chunk = [(2 * rank * m + 15) // 16 * 16 + 48 for m in (n_in, n_out)]
        self.a = M.to_bits(size * rng.standard_normal((cap, rank, n_in)) / np.sqrt(n_in), kind)
        self.b = M.to_bits(rng.standard_normal((cap, n_out, rank)) / np.sqrt(rank), kind)
        off = (np.arange(n + 1) * per).astype(np.uint64)
        units = rng.permutation(cap)[:n * per].astype(np.int32)
        for a in away:
            units[a * per:(a + 1) * per] = -1
        self.unit_of = [int(units[a * per + unit]) if unit < per else -1 for a in range(n)]
        self.bufs = []
        for m, c in zip((self.a, self.b), self.chunk):
            raw = np.full((cap, c), SENTINEL, np.uint8)
            raw[:, :2 * rank * m.size // cap // rank] = m.reshape(cap, -1).view(np.uint8)
            self.bufs.append(up(raw))
        self.bufs += [up(units), up(off)]
        self.desc = B.adapters(units=self.bufs[2].ptr, agent_off=self.bufs[3].ptr, n_agents=n,
                               n_entries=n * per, capacity_units=cap, a=self.bufs[0].ptr,
                               b=self.bufs[1].ptr, a_unit_bytes=self.chunk[0],
                               b_unit_bytes=self.chunk[1], rank=rank, n_in=n_in, n_out=n_out,
                               type=kind, unit=unit)

    def free(self):
        for b in self.bufs:
            b.free()


def run(ad, batch, *, scales=None, in_place=False, pad=0, size=1.0, seed=0, stream=0):
    rng = np.random.default_rng(seed)
    x = Rows(batch.n_rows, 1, ad.n_in, ad.kind, pad=pad,
             values=size * rng.standard_normal((batch.n_rows, 1, ad.n_in)))
    y = rng.standard_normal((batch.n_rows, 1, ad.n_out))
    base = Rows(batch.n_rows, 1, ad.n_out, ad.kind, pad=pad, values=y)
    out = base if in_place else Rows(batch.n_rows, 1, ad.n_out, ad.kind, pad=8 - pad if pad else 0)
    need = B.adapter_add_workspace(ad.desc, batch.n_rows, len(batch.rows))
    ws = DeviceBuffer(max(need, 16))
    d_s = up(np.asarray(scales, np.float32)) if scales is not None else None
    B.adapter_add(ad.desc, batch.desc, x.ptr, base.ptr, out.ptr, x_stride=x.row_stride,
                  base_stride=base.row_stride, out_stride=out.row_stride, workspace=ws.ptr,
                  workspace_bytes=need, scales=d_s.ptr if d_s else 0, stream=stream)
    B.stream_sync(stream)
    got, clean = out.bits()
    assert clean, "bytes outside the rows were written"
    xv, bv = x.before()[:, 0], base.before()[:, 0]
    u = M.HALF_STEP[ad.kind]
    for r in range(len(batch.rows)):
        at = slice(int(batch.row_off[r]), int(batch.row_off[r + 1]))
        a = int(batch.agents[r])
        unit = ad.unit_of[a] if a < len(ad.unit_of) else -1
        if unit < 0:
            assert np.array_equal(got[at, 0], M.to_bits(bv[at], ad.kind)), r
            continue
        s = 1.0 if scales is None else float(np.float32(scales[r]))
        am, bm = M.from_bits(ad.a[unit], ad.kind), M.from_bits(ad.b[unit], ad.kind)
        want, second, first = M.adapter(xv[at], am, bm, bv[at], s)
        tol = u * np.abs(want) + (u * u + (2 * ad.rank + 8) * 2.0 ** -24) * second + \
            (ad.n_in + 40) * 2.0 ** -24 * first + 2.0 ** -23 * np.abs(bv[at])
        if ad.kind == M.F16:
            top = np.abs(xv[at] @ am.T).max(-1, initial=0)[:, None]
            tol = tol + abs(s) * 2.0 ** -24 * top * np.abs(bm).sum(1)[None] + 2.0 ** -25
        value = M.from_bits(got[at, 0], ad.kind)
        assert (np.abs(value - want) <= tol).all(), (r, np.abs(value - want).max(), tol.min())
    n = int(batch.row_off[-1])
    rest = base.view(base.bytes)[n:] if in_place else np.full((batch.n_rows - n, 1, ad.n_out), SENTINEL * 0x101)
    assert np.array_equal(got[n:], rest), "rows behind the last request were written"
    for b in (x, base, out, ws):
        b.free()
    return got


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("rank,n_in,n_out", [(8, 8, 8), (16, 4096, 1000), (16, 264, 4096), (24, 1000, 264),
                                             (32, 2048, 520), (64, 776, 776), (72, 128, 2056),
                                             (128, 520, 1536), (120, 136, 40)])
def test_single_rows(kind, rank, n_in, n_out):
    """Decoding: a row a request, several requests of one adapter, one away, one
    that does not exist."""
    rng = np.random.default_rng(rank + n_in)
    ad = Adapters(rng, 6, rank, n_in, n_out, kind, away=(4,))
    batch = Batch([1] * 9, [0, 3, 3, 1, 4, 0, 5, 77, 2], [0] * 9, spare=2)
    run(ad, batch, scales=rng.uniform(-2, 2, 9), pad=8 if rank == 24 else 0, seed=rank)
    ad.free()


@pytest.mark.parametrize("kind", [M.BF16, M.F16])
@pytest.mark.parametrize("rows", [[0, 1, 15, 16, 17], [33, 0, 64, 2], [100], [1] * 40, [3, 200, 7, 31]])
@pytest.mark.parametrize("rank", [8, 40, 64])
def test_ragged_rows(kind, rows, rank):
    rng = np.random.default_rng(sum(rows) + rank)
    ad = Adapters(rng, 4, rank, 392, 328, kind)
    batch = Batch(rows, rng.integers(0, 4, len(rows)), [0] * len(rows), spare=1)
    run(ad, batch, in_place=rank == 40, seed=rank)


@pytest.mark.parametrize("unit", [0, 2, 3])
def test_a_later_unit_of_an_agent(unit):
    """The projection in one of an agent's several units; unit 3 of 3 does not exist."""
    rng = np.random.default_rng(unit)
    ad = Adapters(rng, 3, 16, 256, 256, M.BF16, per=3, unit=unit, away=(1,))
    run(ad, Batch([2, 1, 5], [2, 1, 0], [0] * 3), scales=[1.0, 2.0, 0.5])


def test_fp16_sums_beyond_the_type():
    """A x of about 2 10^5 passes fp16's range, the outputs do not: 32 bits hold it."""
    rng = np.random.default_rng(2)
    ad = Adapters(rng, 2, 16, 1024, 264, M.F16, size=200.0)
    run(ad, Batch([1, 20], [0, 1], [0, 0]), scales=[1e-3, 1e-3], size=1000.0)


def test_zero_rows_scales_and_nothing():
    rng = np.random.default_rng(3)
    ad = Adapters(rng, 2, 16, 256, 256, M.F16)
    run(ad, Batch([2, 3], [0, 1], [0, 0]), scales=[0.0, 1.0], size=0.0)
    run(ad, Batch([0, 0], [0, 1], [0, 0], spare=4))
    run(ad, Batch([], [], [], spare=4))


def test_many_rows_and_requests():
    rng = np.random.default_rng(4)
    ad = Adapters(rng, 50, 16, 64, 64, M.BF16)
    rows = rng.integers(0, 5, 1500)
    a = run(ad, Batch(rows, rng.integers(0, 50, 1500), [0] * 1500, spare=3), seed=1)
    s = B.Stream()
    b = run(ad, Batch(rows, rng.integers(0, 50, 1500), [0] * 1500, spare=3), seed=1, stream=s.handle)
    assert a.shape == b.shape
    s.close()


def test_offsets_that_break_the_rules_end():
    rng = np.random.default_rng(5)
    ad = Adapters(rng, 3, 16, 64, 64, M.BF16)
    for off in ([0, 4, 2, 6], [0, 100, 3, 6], [5, 6, 0, 6]):
        batch = Batch([2, 2, 2], [0, 1, 2], [0] * 3, spare=2)
        batch.bufs[0].upload(np.array(off, np.uint32))
        x = Rows(8, 1, 64, M.BF16, values=np.ones((8, 1, 64)))
        out = Rows(8, 1, 64, M.BF16, values=np.ones((8, 1, 64)))
        need = B.adapter_add_workspace(ad.desc, 8, 3)
        ws = DeviceBuffer(need)
        B.adapter_add(ad.desc, batch.desc, x.ptr, out.ptr, out.ptr, x_stride=64, base_stride=64,
                      out_stride=64, workspace=ws.ptr, workspace_bytes=need)
        B.null_stream_sync()
        assert out.bits()[1]
