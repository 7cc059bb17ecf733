"""ss_kv_write and ss_kv_read against the plain forms in 64 bits: layouts, page
sizes, types, ragged batches, agents that are away, rows of nobody, and what
is beside the written bytes."""
import numpy as np
import pytest

from model_harness import SENTINEL, Batch, Cache, Rows
from oracle import model as M
from paper_2601_21473_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert B.device_count() > 0, "GPU tests need a GPU"


CASES = [   # page, heads, dim, order, gap, rows, lens (after the step)
    (16, 8, 128, "head", 0, [1, 1, 1], [1, 17, 33]),
    (16, 2, 64, "token", 0, [256], [256]),
    (1, 1, 16, "head", 0, [5, 0, 3], [5, 2, 9]),
    (4, 3, 80, "token", 16, [7, 1, 30, 2], [8, 1, 41, 2]),
    (64, 1, 256, "head", 32, [63, 65, 2], [63, 70, 129]),
    (32, 5, 144, "token", 0, [3, 40], [50, 40]),
    (1024, 2, 48, "head", 0, [10, 1100], [1500, 1100]),
    (16, 4, 112, "head", 16, [1] * 70, list(range(1, 71))),
    (16, 1, 128, "token", 0, [1500, 1, 900], [1500, 16, 901]),
]


def case(i, kind, away=()):
    page, heads, dim, order, gap, rows, lens = CASES[i]
    rng = np.random.default_rng(100 + i)
    cache = Cache(rng, list(lens) + [5], page=page, heads=heads, dim=dim, kind=kind, order=order,
                  gap=gap, away=away, scale_gap=16 * (i % 2))
    batch = Batch(rows, np.arange(len(rows)), lens, spare=2)
    return rng, cache, batch


def new_rows(rng, batch, cache, kind, pad, by_head):
    out = []
    for _ in range(2):
        x = rng.standard_normal((batch.n_rows, cache.heads, cache.dim)) * \
            2.0 ** rng.integers(-20, 12, (batch.n_rows, cache.heads, 1))
        out.append(Rows(batch.n_rows, cache.heads, cache.dim, kind, values=x, pad=pad, by_head=by_head))
    return out


def check_write(cache, batch, new, before):
    """Every byte of the planes: the batch's tokens hold the rows, all else is as
    it was.  Codes are the nearest to the quotient in 64 bits within the 32-bit
    division's rounding (2^-24 of it)."""
    request, token = M.positions(batch.row_off, batch.lens)
    got = cache.download()
    for i in range(2):
        x = M.from_bits(new[i].view(new[i].bytes).copy(), new[i].kind)
        want = before[i].copy()
        body, scales = cache.body(want), cache.scale_view(want) if cache.kind == M.E4M3 else None
        for t in range(len(request)):
            at = cache.place(int(batch.agents[request[t]]), int(token[t]))
            if at is None:
                continue
            u, slot = at
            if cache.kind != M.E4M3:
                body[u, :, slot] = new[i].view(new[i].bytes)[t]
                continue
            s = M.e4m3_scale(x[t])
            scales[u, :, slot] = s
            codes = cache.body(got[i])[u, :, slot]
            q = x[t] / s[:, None].astype(np.float64)
            v = M.from_bits(codes, M.E4M3)
            nan = np.isnan(q)
            assert (np.isnan(v) == nan).all()
            q = np.clip(q, -448, 448)
            ok = np.abs(v - q) <= M.e4m3_half_step(q) + 2.0 ** -24 * np.abs(q)
            assert ok[~nan].all()
            # ties of the 32-bit quotient go to the even code
            q32 = np.clip((x[t].astype(np.float32) / s[:, None]).astype(np.float64), -448, 448)
            tie = ~nan & (np.abs(v - q32) == M.e4m3_half_step(q32)) & (np.abs(q32) < 448)
            assert (codes[tie] % 2 == 0).all()
            body[u, :, slot] = codes
        assert np.array_equal(got[i], want), "bytes that no row goes to were written"


@pytest.mark.parametrize("kind,rows_kind", [(M.BF16, M.BF16), (M.F16, M.F16), (M.E4M3, M.BF16),
                                            (M.E4M3, M.F16)])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_write(i, kind, rows_kind):
    rng, cache, batch = case(i, kind, away=(1,) if i % 3 == 2 else ())
    new = new_rows(rng, batch, cache, rows_kind, pad=8 * (i % 3), by_head=i % 2 == 1)
    before = [b.copy() for b in cache.bytes]
    B.kv_write(cache.desc, batch.desc, new[0].ptr, new[1].ptr, type=rows_kind, strides=new[0].strides)
    B.null_stream_sync()
    check_write(cache, batch, new, before)
    for x in [cache, batch] + new:
        x.free()


@pytest.mark.parametrize("rows_kind", [M.BF16, M.F16])
def test_write_of_zeros_infinities_and_nan(rows_kind):
    rng, cache, batch = case(0, M.E4M3)
    x = rng.standard_normal((batch.n_rows, cache.heads, cache.dim))
    x[0, 0] = 0
    x[0, 1] = -0.0
    x[0, 2, 5] = np.inf
    x[0, 3, 7] = -np.inf
    x[0, 4, ::2] = np.nan
    x[0, 5] = np.nan
    x[0, 6] = np.inf
    x[0, 7] = 0
    x[0, 7, 3] = 2.0 ** -24 if rows_kind == M.F16 else 2.0 ** -133      # smallest of the type
    x[1] = 65504 if rows_kind == M.F16 else 3.3e38
    new = [Rows(batch.n_rows, cache.heads, cache.dim, rows_kind, values=v) for v in (x, x[:, ::-1])]
    before = [b.copy() for b in cache.bytes]
    B.kv_write(cache.desc, batch.desc, new[0].ptr, new[1].ptr, type=rows_kind, strides=new[0].strides)
    B.null_stream_sync()
    check_write(cache, batch, new, before)


@pytest.mark.parametrize("kind,rows_kind", [(M.BF16, M.BF16), (M.F16, M.F16), (M.E4M3, M.BF16),
                                            (M.E4M3, M.F16)])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_read(i, kind, rows_kind):
    rng, cache, batch = case(i, kind, away=(1,) if i % 3 == 1 else ())
    out = [Rows(batch.n_rows, cache.heads, cache.dim, rows_kind, pad=8 * (i % 3), by_head=i % 2 == 0)
           for _ in range(2)]
    B.kv_read(cache.desc, batch.desc, out[0].ptr, out[1].ptr, type=rows_kind, strides=out[0].strides)
    B.null_stream_sync()
    request, token = M.positions(batch.row_off, batch.lens)
    n = len(request)
    stored = {a: cache.tokens(a, int(batch.lens[a])) for a in range(len(batch.rows))}
    for w in range(2):
        got, clean = out[w].bits()
        assert clean
        assert (got[n:] == SENTINEL * 0x101).all(), "rows behind the last request were written"
        want = np.stack([stored[request[t]][w][token[t]] for t in range(n)])
        value = M.from_bits(got[:n], rows_kind)
        # the product in 32 bits, then the type's rounding (fp16: also below 2^-14)
        tol = 0 if kind != M.E4M3 else np.abs(want) * (M.HALF_STEP[rows_kind] + 2.0 ** -24) + \
            (2.0 ** -25 if rows_kind == M.F16 else 0)
        assert (np.abs(value - want) <= tol).all()
        away = np.array([not stored[request[t]][2][token[t]] for t in range(n)])
        assert (got[:n][away] == 0).all()


def test_tokens_before_the_first_and_behind_the_pages():
    """lens below a request's rows: the early rows have no token.  Tokens behind an
    agent's pages and agents that do not exist: not written, read as zeros."""
    rng = np.random.default_rng(7)
    cache = Cache(rng, [20, 16, 3], page=16, heads=2, dim=64, kind=M.BF16)
    batch = Batch([5, 4, 2, 3, 1], [0, 1, 2, 9, 0xFFFFFFFF], [3, 18, 0, 5, 1])
    new = new_rows(rng, batch, cache, M.BF16, 0, False)
    before = [b.copy() for b in cache.bytes]
    B.kv_write(cache.desc, batch.desc, new[0].ptr, new[1].ptr, type=M.BF16, strides=new[0].strides)
    out = [Rows(batch.n_rows, 2, 64, M.BF16) for _ in range(2)]
    B.kv_read(cache.desc, batch.desc, out[0].ptr, out[1].ptr, type=M.BF16, strides=out[0].strides)
    B.null_stream_sync()
    check_write(cache, batch, new, before)
    request, token = M.positions(batch.row_off, batch.lens)
    for w in range(2):
        got, clean = out[w].bits()
        assert clean
        for t in range(len(request)):
            there = cache.place(int(batch.agents[request[t]]), int(token[t])) is not None
            assert np.array_equal(got[t], new[w].view(new[w].bytes)[t] if there else got[t] * 0), t


def test_empty_batches_do_nothing():
    rng = np.random.default_rng(8)
    cache = Cache(rng, [20], page=16, heads=2, dim=64, kind=M.E4M3)
    new = [Rows(3, 2, 64, M.BF16, values=np.ones((3, 2, 64))) for _ in range(2)]
    for batch in (Batch([0, 0], [0, 0], [5, 6], spare=3), Batch([], [], [], spare=3)):
        B.kv_write(cache.desc, batch.desc, new[0].ptr, new[1].ptr, type=M.BF16, strides=new[0].strides)
        B.kv_read(cache.desc, batch.desc, new[0].ptr, new[1].ptr, type=M.BF16, strides=new[0].strides)
    B.null_stream_sync()
    assert all(np.array_equal(a, b) for a, b in zip(cache.download(), cache.bytes))
    assert all((r.values() == 1).all() for r in new)


@pytest.mark.parametrize("kind", [M.BF16, M.E4M3])
def test_units_beyond_4_gib(kind):
    """A plane of more than 4 GiB: the last units are written and read where they are."""
    heads, dim, page = 8, 128, 16
    chunk = 4 << 20
    cap = 1100                                       # 4.6 GB a plane
    size = 1 if kind == M.E4M3 else 2
    from model_harness import up
    from paper_2601_21473_amd.memory import DeviceBuffer
    planes = [DeviceBuffer(cap * chunk) for _ in range(2)]
    units = np.array([cap - 1, 1030, 0], np.int32)
    off = np.array([0, 3], np.uint64)
    d_units, d_off = up(units), up(off)
    desc = B.kv_cache(units=d_units.ptr, agent_off=d_off.ptr, n_agents=1, n_entries=3,
                      capacity_units=cap, k=planes[0].ptr, v=planes[1].ptr, k_unit_bytes=chunk,
                      v_unit_bytes=chunk, page_tokens=page, n_heads=heads, head_dim=dim, type=kind,
                      token_bytes=dim * size, head_bytes=page * dim * size,
                      scale_off=page * heads * dim if kind == M.E4M3 else 0)
    rng = np.random.default_rng(9)
    batch = Batch([40], [0], [40])
    # values that every type holds exactly: powers of two below the largest, 448
    x = 448.0 * 2.0 ** -rng.integers(0, 6, (40, heads, dim))
    x[:, :, 0] = 448
    new = [Rows(40, heads, dim, M.BF16, values=v) for v in (x, -x)]
    out = [Rows(40, heads, dim, M.BF16) for _ in range(2)]
    B.kv_write(desc, batch.desc, new[0].ptr, new[1].ptr, type=M.BF16, strides=new[0].strides)
    B.kv_read(desc, batch.desc, out[0].ptr, out[1].ptr, type=M.BF16, strides=out[0].strides)
    B.null_stream_sync()
    assert np.array_equal(out[0].values(), x) and np.array_equal(out[1].values(), -x)
    for u, t in ((cap - 1, 0), (1030, 16), (0, 32)):
        raw = planes[0].download(u * chunk, dim * size)
        v = M.from_bits(raw if kind == M.E4M3 else raw.view(np.uint16), kind)
        assert np.array_equal(v, x[t, 0])
    for b in planes:
        b.free()
