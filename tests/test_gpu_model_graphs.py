"""The operators over resident units with a framework's memory and streams: captured
into graphs and replayed with new lengths and contents, eager calls in between, and
two streams at once with workspaces of their own.  In a child process, as the
framework brings its own copy of the HIP runtime, which has to be loaded first."""
import os
import subprocess
import sys

import pytest

from paper_2601_21473_amd import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import sys
import torch
from paper_2601_21473_amd import binding as B

DEV = "cuda"
H, PER, D, PAGE, R, RANK, NIN, NOUT = 2, 4, 128, 16, 9, 16, 256, 512
kind = int(sys.argv[1])
g = torch.Generator(device=DEV).manual_seed(5)
rnd = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
MOST, PREFIX = 40, 70                                   # pages of an agent, of the prefix
pages = torch.tensor([MOST] * R + [PREFIX], device=DEV)
off = torch.cat([pages.new_zeros(1), pages.cumsum(0)])
total = int(off[-1])
units = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
size = 1 if kind == B.SS_E4M3 else 2
body = PAGE * H * D * size
chunk = body + (4 * PAGE * H if size == 1 else 0)


class Call:
    """A step's buffers: lengths and contents change, addresses stay."""

    def __init__(self):
        self.planes = [torch.zeros(total * chunk, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.cache = B.kv_cache(units=units.data_ptr(), agent_off=off.data_ptr(), n_agents=R + 1,
                                n_entries=total, capacity_units=total, k=self.planes[0].data_ptr(),
                                v=self.planes[1].data_ptr(), k_unit_bytes=chunk, v_unit_bytes=chunk,
                                page_tokens=PAGE, n_heads=H, head_dim=D, type=kind,
                                token_bytes=D * size, head_bytes=PAGE * D * size,
                                scale_off=body if size == 1 else 0)
        self.row_off, self.agents = i32(list(range(R + 1))), i32(list(range(R)))
        self.lens = i32([1] * R)
        self.groups = (i32([0, R - 2]), i32([R]), i32([1]))
        self.batch = B.batch(n_rows=R, n_requests=R, row_off=self.row_off.data_ptr(),
                             agents=self.agents.data_ptr(), lens=self.lens.data_ptr(), n_groups=1,
                             group_off=self.groups[0].data_ptr(),
                             prefix_agents=self.groups[1].data_ptr(),
                             prefix_lens=self.groups[2].data_ptr())
        self.k, self.v = rnd(R, H, D), rnd(R, H, D)
        self.q, self.out = rnd(R, H * PER, D), rnd(R, H * PER, D)
        self.lse = torch.zeros(R, H * PER, device=DEV)
        self.back = [rnd(R, H, D) for _ in range(2)]
        self.a, self.b = rnd(total, RANK, NIN) / 16, rnd(total, NOUT, RANK) / 4
        self.ad = B.adapters(units=units.data_ptr(), agent_off=off.data_ptr(), n_agents=R + 1,
                             n_entries=total, capacity_units=total, a=self.a.data_ptr(),
                             b=self.b.data_ptr(), a_unit_bytes=RANK * NIN * 2,
                             b_unit_bytes=RANK * NOUT * 2, rank=RANK, n_in=NIN, n_out=NOUT,
                             type=B.SS_BF16, unit=3)
        self.x, self.base = rnd(R, NIN), rnd(R, NOUT)
        self.y = torch.empty_like(self.base)
        need = max(B.prefix_attention_workspace(self.cache, self.batch, H * PER),
                   B.adapter_add_workspace(self.ad, R, R))
        self.ws = torch.empty(need, dtype=torch.uint8, device=DEV)

    def new(self):
        """New lengths, a new past, new rows."""
        n = torch.randint(1, MOST * PAGE + 1, (R,), generator=g, device=DEV)
        self.lens.copy_(n)
        self.groups[2].copy_(torch.randint(1, PREFIX * PAGE + 1, (1,), generator=g, device=DEV))
        for p in self.planes:
            if size == 2:
                p.view(torch.bfloat16).copy_(rnd(p.numel() // 2))
            else:
                codes = torch.randint(0, 120, (total, chunk), generator=g, device=DEV).to(torch.uint8)
                codes[:, body:] = (torch.rand(total, PAGE * H, generator=g, device=DEV) * 0.01 + 0.001
                                   ).view(torch.uint8)
                p.copy_(codes.view(-1))
        for t in (self.k, self.v, self.q, self.x, self.base):
            t.copy_(rnd(*t.shape))

    def run(self):
        s = torch.cuda.current_stream().cuda_stream
        B.kv_write(self.cache, self.batch, self.k.data_ptr(), self.v.data_ptr(), type=B.SS_BF16,
                   strides=(H * D, D), stream=s)
        B.prefix_attention(self.cache, self.batch, self.q.data_ptr(), self.out.data_ptr(),
                           type=B.SS_BF16, n_q_heads=H * PER, q_strides=(H * PER * D, D),
                           out_strides=(H * PER * D, D), scale=D ** -0.5, lse=self.lse.data_ptr(),
                           workspace=self.ws.data_ptr(), workspace_bytes=self.ws.numel(), stream=s)
        B.kv_read(self.cache, self.batch, self.back[0].data_ptr(), self.back[1].data_ptr(),
                  type=B.SS_BF16, strides=(H * D, D), stream=s)
        B.adapter_add(self.ad, self.batch, self.x.data_ptr(), self.base.data_ptr(), self.y.data_ptr(),
                      x_stride=NIN, base_stride=NOUT, out_stride=NOUT, workspace=self.ws.data_ptr(),
                      workspace_bytes=self.ws.numel(), stream=s)

    def results(self):
        return [t.clone() for t in (self.out, self.lse, *self.back, self.y, *self.planes)]


def same(a, b, what):
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (what, i)


calls = [Call(), Call()]
for c in calls:
    c.new()
    c.run()
torch.cuda.synchronize()
# each call captured with its own buffers and workspace
graphs = []
for c in calls:
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    graphs.append(graph)
for turn in range(4):
    want = []
    for c in calls:
        c.new()
        c.run()                                          # eager, as the oracle of the replay
        want.append(c.results())
        for t in (c.out, c.lse, c.y, *c.back):
            t.zero_()
    torch.cuda.synchronize()
    for i in (0, 1) if turn % 2 else (1, 0):
        graphs[i].replay()
        if turn == 2:
            graphs[i].replay()
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        same(c.results(), w, ("replay", turn))
    assert all(torch.isfinite(c.out).all() for c in calls)
    print("turn", turn, "ok", flush=True)
# both at once on two streams
streams = [torch.cuda.Stream(), torch.cuda.Stream()]
for turn in range(3):
    want = []
    for c in calls:
        c.new()
        c.run()
        want.append(c.results())
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c.run()
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        same(c.results(), w, ("streams", turn))
print("CHILD OK", flush=True)
'''


@pytest.mark.parametrize("kind", [B.SS_BF16, B.SS_E4M3])
def test_graphs_and_streams(kind):
    pytest.importorskip("torch")
    env = dict(os.environ, PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-u", "-c", CHILD, str(kind)], env=env, cwd=ROOT,
                       capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "CHILD OK" in r.stdout, r.stdout[-1500:] + r.stderr[-2500:]
