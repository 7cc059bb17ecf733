"""The operators together, as a program uses them: pools of KV pages and adapters
are planned and moved, a step's keys and values are written into the pages the plan
made resident, attention runs over them and over shared prefixes (objects of the same
pool), and the agents' adapters are added to a projection.  Agents come and go
between steps, so most tokens that a step sees have been evicted and loaded again."""
import numpy as np
import pytest

from model_harness import Batch, Rows, up
from oracle import model as M
from paper_2601_21473_amd import binding as B
from paper_2601_21473_amd.memory import DeviceBuffer, PoolMemory
from test_gpu_adapters import run as run_adapters
from test_gpu_prefix_attention import attend, check
from workloads.traces import PoolSpec

pytestmark = pytest.mark.gpu

N, PREFIXES, PAGE, HEADS, DIM, PER = 10, 2, 16, 2, 64, 2
RANK, N_IN, N_OUT = 16, 256, 392


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert B.device_count() > 0, "GPU tests need a GPU"


class Layer:
    """What test_gpu_prefix_attention.check needs of a cache, kept on the host."""

    def __init__(self, desc, kind, pages):
        self.desc, self.kind, self.page, self.heads, self.dim = desc, kind, PAGE, HEADS, DIM
        self.off = np.concatenate([[0], np.cumsum(pages)]).astype(np.int64)
        self.lens = np.zeros(len(pages), np.int64)
        self.kv = [[np.zeros((int(p) * PAGE, HEADS, DIM)) for p in pages] for _ in range(2)]

    def tokens(self, agent, count):
        return self.kv[0][agent][:count], self.kv[1][agent][:count], np.ones(count, bool)


class PoolAdapters:
    def __init__(self, desc, a, b, kind, n):
        self.desc, self.a, self.b, self.kind = desc, a, b, kind
        self.rank, self.n_in, self.n_out = RANK, N_IN, N_OUT
        self.unit_of = list(range(n))               # a and b are indexed by agent here


@pytest.mark.parametrize("kind,rows_kind,order,direct", [
    (M.BF16, M.BF16, "head", 0), (M.E4M3, M.BF16, "token", 1 << 22), (M.F16, M.F16, "head", 1 << 22),
    (M.E4M3, M.F16, "head", 0)])
def test_steps_of_a_simulation(kind, rows_kind, order, direct):
    rng = np.random.default_rng(kind * 10 + rows_kind)
    size = 1 if kind == M.E4M3 else 2
    page_bytes = HEADS * PAGE * (DIM * size + (4 if size == 1 else 0))
    chunk = page_bytes + 64                          # the layer lies 64 bytes into its chunk
    pages = np.array([4] * N + [6, 9], np.uint32)
    total = N + PREFIXES
    spec = PoolSpec("kv", 4 * 4 + 15 + 2, [chunk] * 4, pages)       # room for 4 agents
    mem = PoolMemory(spec, 2 * 2 * 8 * spec.unit_bytes, 2)
    mem.host_np[:] = 0
    pool = mem.make_pool(direct_bytes=direct)
    layers = [Layer(pool.kv_cache(2 * i, 2 * i + 1, page_tokens=PAGE, n_heads=HEADS, head_dim=DIM,
                                  type=kind, order=order, k_offset=64, v_offset=32), kind, pages)
              for i in range(2)]
    aspec = PoolSpec("adapters", 4, [2 * RANK * N_IN, 2 * RANK * N_OUT], np.ones(N, np.uint32))
    amem = PoolMemory(aspec, 2 * 2 * aspec.unit_bytes, 2)
    a_bits = M.to_bits(rng.standard_normal((N, RANK, N_IN)) / 16, rows_kind)
    b_bits = M.to_bits(rng.standard_normal((N, N_OUT, RANK)) / 4, rows_kind)
    for a in range(N):
        amem.host_copy(a)[:] = np.concatenate([a_bits[a].reshape(-1).view(np.uint8),
                                               b_bits[a].reshape(-1).view(np.uint8)])
    apool = amem.make_pool(direct_bytes=direct)
    adapters = PoolAdapters(apool.adapters(0, 1, rank=RANK, n_in=N_IN, n_out=N_OUT, type=rows_kind),
                            a_bits, b_bits, rows_kind, N)
    d_dist, d_act, d_adist, d_aact = (DeviceBuffer(4 * total) for _ in range(4))
    stream = B.Stream()
    shared_by = {0: range(0, 5), 1: range(5, 8)}     # agents 8 and 9 share nothing
    evicted = 0
    for step in range(14):
        if step < PREFIXES:                          # the prefixes are computed first
            active = [N + step]
            rows = [int(pages[N + step]) * PAGE - 3]
            groups = None
        else:
            active = sorted(rng.choice(N, 4, replace=False).tolist())
            rows = [int(min(rng.choice([1, 1, 2, 9]), pages[a] * PAGE - layers[0].lens[a])) for a in active]
            off, pa = [0], []
            for g, members in shared_by.items():
                off.append(off[-1] + sum(a in members for a in active))
                pa.append(N + g)
            groups = (off, pa, [int(layers[0].lens[p]) for p in pa])
        mask = np.zeros(total, np.uint8)
        mask[active] = 1
        if groups:
            mask[N:] = 1
        dist = np.where(mask == 1, 0, rng.integers(1, 30, total)).astype(np.uint32)
        d_dist.upload(dist)
        d_act.upload(mask)
        d_adist.upload(dist[:N])
        d_aact.upload(mask[:N])
        for p, d, m in ((pool, d_dist, d_act), (apool, d_adist, d_aact)):
            plan = p.plan_step(d.ptr, m.ptr, 4, None, stream.handle)
            evicted += plan["n_victims"]
            p.evict_pack(stream.handle)
            p.prefetch_unpack(stream.handle)
        lens = [int(layers[0].lens[a]) + r for a, r in zip(active, rows)]
        batch = Batch(rows, active, lens, groups, spare=1)
        request, token = M.positions(batch.row_off, batch.lens)
        for layer in layers:
            new = [Rows(batch.n_rows, HEADS, DIM, rows_kind,
                        values=rng.standard_normal((batch.n_rows, HEADS, DIM))) for _ in range(2)]
            B.kv_write(layer.desc, batch.desc, new[0].ptr, new[1].ptr, type=rows_kind,
                       strides=new[0].strides, stream=stream.handle)
            for i in range(2):
                held = M.stored(new[i].before(), kind)
                for t in range(len(request)):
                    layer.kv[i][active[request[t]]][token[t]] = held[t]
            layer.lens[active] = lens
            q = Rows(batch.n_rows, HEADS * PER, DIM, rows_kind,
                     values=rng.standard_normal((batch.n_rows, HEADS * PER, DIM)))
            got, lse = attend(layer, batch, q, PER, rows_kind, scale=0.125, stream=stream.handle)
            check(layer, batch, q, PER, rows_kind, got, lse, 0.125)
            for x in new + [q]:
                x.free()
        if groups:
            run_adapters(adapters, Batch(rows, active, lens, spare=1), seed=step, stream=stream.handle,
                         scales=rng.uniform(0.5, 2, len(rows)))
    assert evicted > 10
    # what the pool wrote back and still holds: every agent's tokens, in its pages
    whole = [a for a in range(total) if layers[0].lens[a] and pool.resident_host()[a]]
    batch = Batch([int(layers[0].lens[a]) for a in whole], whole, [int(layers[0].lens[a]) for a in whole])
    for layer in layers:
        out = [Rows(batch.n_rows, HEADS, DIM, rows_kind) for _ in range(2)]
        B.kv_read(layer.desc, batch.desc, out[0].ptr, out[1].ptr, type=rows_kind,
                  strides=out[0].strides, stream=stream.handle)
        stream.sync()
        for i in range(2):
            want = np.concatenate([layer.kv[i][a][:int(layer.lens[a])] for a in whole])
            tol = np.abs(want) * (M.HALF_STEP[rows_kind] + 2.0 ** -24) + 2.0 ** -25 if size == 1 else 0
            assert (np.abs(out[i].values() - want) <= tol).all()
    pool.sync()
    pool.close()
    apool.close()
    stream.close()
    mem.free()
    amem.free()
