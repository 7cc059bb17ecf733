"""The operators over resident units called by several host threads at once, each with a
stream, a workspace and outputs of its own, between calls that are refused."""
import threading

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


class Caller:
    """One thread's batch over the shared cache and adapters, and what its calls give alone."""

    def __init__(self, seed, cache, ad, rows, agents, prefix):
        rng = np.random.default_rng(seed)
        self.cache, self.ad, self.rng = cache, ad, rng
        lens = [int(cache.lens[a]) for a in agents]
        self.batch = Batch(rows, agents, lens, ([0, len(rows)], [prefix], [int(cache.lens[prefix])]))
        n = self.n = self.batch.n_rows
        self.q = Rows(n, 8, 64, M.BF16, values=rng.standard_normal((n, 8, 64)))
        self.x = Rows(n, 1, ad.n_in, M.BF16, values=rng.standard_normal((n, 1, ad.n_in)))
        self.base = Rows(n, 1, ad.n_out, M.BF16, values=rng.standard_normal((n, 1, ad.n_out)))
        self.stream = B.Stream()
        self.need = [B.prefix_attention_workspace(cache.desc, self.batch.desc, 8),
                     B.adapter_add_workspace(ad.desc, n, len(rows))]
        self.ws = [DeviceBuffer(max(x, 16)) for x in self.need]
        got, lse = attend(cache, self.batch, self.q, 4, M.BF16, scale=0.125)
        check(cache, self.batch, self.q, 4, M.BF16, got, lse, 0.125)
        self.want = self.outputs()
        self.call(self.want, 0)
        B.null_stream_sync()
        self.want_bits = [r.bits()[0] for r in self.want]
        assert np.array_equal(self.want_bits[0], got)
        self.error = None

    def outputs(self):
        return [Rows(self.n, 8, 64, M.BF16), Rows(self.n, 1, self.ad.n_out, M.BF16),
                Rows(self.n, 2, 64, M.BF16), Rows(self.n, 2, 64, M.BF16)]

    def call(self, out, stream):
        c, b = self.cache.desc, self.batch.desc
        B.prefix_attention(c, b, self.q.ptr, out[0].ptr, type=M.BF16, n_q_heads=8, q_strides=self.q.strides,
                           out_strides=out[0].strides, scale=0.125, workspace=self.ws[0].ptr,
                           workspace_bytes=self.need[0], stream=stream)
        B.adapter_add(self.ad.desc, b, self.x.ptr, self.base.ptr, out[1].ptr, x_stride=self.x.row_stride,
                      base_stride=self.base.row_stride, out_stride=out[1].row_stride,
                      workspace=self.ws[1].ptr, workspace_bytes=self.need[1], stream=stream)
        B.kv_read(c, b, out[2].ptr, out[3].ptr, type=M.BF16, strides=out[2].strides, stream=stream)

    def work(self, start, refusal):
        try:
            outs = [self.outputs() for _ in range(20)]
            start.wait(30)
            for out in outs:
                self.call(out, self.stream.handle)
                with pytest.raises(B.ScaleSimError, match=refusal[0]):
                    refusal[1](self)
            self.stream.sync()
            for i, out in enumerate(outs):
                for r, want in zip(out, self.want_bits):
                    got, clean = r.bits()
                    assert clean and np.array_equal(got, want), i
        except BaseException as e:                   # told by the test's own thread
            self.error = e


def refuse_workspace(c):
    B.adapter_add(c.ad.desc, c.batch.desc, c.x.ptr, c.base.ptr, c.base.ptr, x_stride=c.x.row_stride,
                  base_stride=c.base.row_stride, out_stride=c.base.row_stride, workspace=c.ws[1].ptr,
                  workspace_bytes=0)


def refuse_heads(c):
    B.prefix_attention(c.cache.desc, c.batch.desc, c.q.ptr, c.q.ptr, type=M.BF16, n_q_heads=7,
                       q_strides=c.q.strides, out_strides=c.q.strides, scale=1.0, workspace=c.ws[0].ptr,
                       workspace_bytes=c.need[0])


def refuse_type(c):
    B.kv_read(c.cache.desc, c.batch.desc, c.q.ptr, c.q.ptr, type=M.F16, strides=c.q.strides)


def test_three_threads():
    rng = np.random.default_rng(0)
    cache = Cache(rng, [100, 40, 300, 65, 128, 700], page=16, heads=2, dim=64, kind=M.BF16)
    ad = Adapters(rng, 6, 16, 256, 520, M.BF16, away=(3,))
    callers = [Caller(1, cache, ad, [1, 1, 1], [0, 1, 2], 5), Caller(2, cache, ad, [20, 40], [3, 4], 5),
               Caller(3, cache, ad, [1, 2, 3, 1], [4, 0, 2, 3], 1)]
    refusals = [("workspace_bytes", refuse_workspace), ("n_q_heads", refuse_heads), ("with a cache", refuse_type)]
    start = threading.Barrier(len(callers))
    threads = [threading.Thread(target=c.work, args=(start, r)) for c, r in zip(callers, refusals)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(100)
    assert not any(t.is_alive() for t in threads)
    for c in callers:
        if c.error is not None:
            raise c.error
        c.stream.close()
