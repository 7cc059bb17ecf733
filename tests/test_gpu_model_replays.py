"""Replayed graphs and concurrent streams of the operators over resident units, with
everything they write cleared before: outputs hold a sentinel and the planes their contents
from before the step's tokens, every replay and every concurrent call has outputs and
planes of its own that are compared, and the eager result is compared with the 64-bit form.
In a child process, as the framework brings its own copy of the HIP runtime."""
import os
import subprocess
import sys

import pytest

from paper_2601_21473_amd import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import sys
import numpy as np
import torch
from oracle import model as M
from paper_2601_21473_amd import binding as B

DEV = "cuda"
H, PER, D, PAGE, R, RANK, NIN, NOUT = 2, 4, 64, 16, 7, 16, 128, 264
kind, ROWS = int(sys.argv[1]), [1] * R if sys.argv[2] == "decode" else [1, 9, 2, 30, 1, 5, 0]
T, RUNS = sum(ROWS), 5
g = torch.Generator(device=DEV).manual_seed(7)
rnd = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
MOST, PREFIX = 8, 20                                    # pages of an agent, of the prefix
pages = [MOST] * R + [PREFIX]
off = torch.tensor(np.concatenate([[0], np.cumsum(pages)]), dtype=torch.int64, device=DEV)
total = int(off[-1])
units = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
size = 1 if kind == B.SS_E4M3 else 2
body = PAGE * H * D * size
chunk = body + (4 * PAGE * H if size == 1 else 0)


class Run:
    """What one call of the four operators writes, and its workspaces."""

    def __init__(self, c):
        self.planes = [torch.empty(total * chunk, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.cache = B.kv_cache(units=units.data_ptr(), agent_off=off.data_ptr(), n_agents=R + 1,
                                n_entries=total, capacity_units=total, k=self.planes[0].data_ptr(),
                                v=self.planes[1].data_ptr(), k_unit_bytes=chunk, v_unit_bytes=chunk,
                                page_tokens=PAGE, n_heads=H, head_dim=D, type=kind,
                                token_bytes=D * size, head_bytes=PAGE * D * size,
                                scale_off=body if size == 1 else 0)
        self.out = torch.empty(T, H * PER, D, device=DEV, dtype=torch.bfloat16)
        self.lse = torch.empty(T, H * PER, device=DEV)
        self.back = [torch.empty(T, H, D, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
        self.y = torch.empty(T, NOUT, device=DEV, dtype=torch.bfloat16)
        need = (B.prefix_attention_workspace(self.cache, c.batch, H * PER), B.adapter_add_workspace(c.ad, T, R))
        self.ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in need]

    def clear(self, c):
        for p, past in zip(self.planes, c.past):
            p.copy_(past)
        for t in (self.out, self.lse, *self.back, self.y):
            t.view(torch.uint8).fill_(0xA5)
        for w in self.ws:
            w.fill_(0xFF)

    def results(self):
        return [t.clone() for t in (self.out, self.lse, *self.back, self.y, *self.planes)]


class Step:
    """A step's inputs, changed in place."""

    def __init__(self):
        self.row_off, self.agents = i32(np.concatenate([[0], np.cumsum(ROWS)])), i32(list(range(R)))
        self.lens, self.groups = i32([1] * R), (i32([0, R - 2]), i32([R]), i32([1]))
        self.batch = B.batch(n_rows=T, n_requests=R, row_off=self.row_off.data_ptr(),
                             agents=self.agents.data_ptr(), lens=self.lens.data_ptr(), n_groups=1,
                             group_off=self.groups[0].data_ptr(), prefix_agents=self.groups[1].data_ptr(),
                             prefix_lens=self.groups[2].data_ptr())
        self.past = [torch.zeros(total * chunk, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.k, self.v, self.q = rnd(T, H, D), rnd(T, H, D), rnd(T, H * PER, D)
        self.a, self.b = rnd(total, RANK, NIN) / 8, rnd(total, NOUT, RANK) / 4
        self.ad = B.adapters(units=units.data_ptr(), agent_off=off.data_ptr(), n_agents=R + 1,
                             n_entries=total, capacity_units=total, a=self.a.data_ptr(),
                             b=self.b.data_ptr(), a_unit_bytes=RANK * NIN * 2, b_unit_bytes=RANK * NOUT * 2,
                             rank=RANK, n_in=NIN, n_out=NOUT, type=B.SS_BF16, unit=3)
        self.x, self.base = rnd(T, NIN), rnd(T, NOUT)

    def new(self):
        n = torch.tensor(ROWS, device=DEV)
        self.lens.copy_(n + (torch.rand(R, generator=g, device=DEV) * (MOST * PAGE - n)).int())
        self.groups[2].copy_(torch.randint(1, PREFIX * PAGE + 1, (1,), generator=g, device=DEV))
        for p in self.past:
            if size == 2:
                p.view(torch.bfloat16).copy_(rnd(p.numel() // 2))
            else:
                codes = torch.randint(0, 120, (total, chunk), generator=g, device=DEV).to(torch.uint8)
                codes[:, body:] = (torch.rand(total, PAGE * H, generator=g, device=DEV) * 0.01 + 0.001
                                   ).view(torch.uint8)
                p.copy_(codes.view(-1))
        for t in (self.k, self.v, self.q, self.x, self.base):
            t.copy_(rnd(*t.shape))

    def call(self, r):
        s = torch.cuda.current_stream().cuda_stream
        B.kv_write(r.cache, self.batch, self.k.data_ptr(), self.v.data_ptr(), type=B.SS_BF16,
                   strides=(H * D, D), stream=s)
        B.prefix_attention(r.cache, self.batch, self.q.data_ptr(), r.out.data_ptr(), type=B.SS_BF16,
                           n_q_heads=H * PER, q_strides=(H * PER * D, D), out_strides=(H * PER * D, D),
                           scale=D ** -0.5, lse=r.lse.data_ptr(), workspace=r.ws[0].data_ptr(),
                           workspace_bytes=r.ws[0].numel(), stream=s)
        B.kv_read(r.cache, self.batch, r.back[0].data_ptr(), r.back[1].data_ptr(), type=B.SS_BF16,
                  strides=(H * D, D), stream=s)
        B.adapter_add(self.ad, self.batch, self.x.data_ptr(), self.base.data_ptr(), r.y.data_ptr(),
                      x_stride=NIN, base_stride=NOUT, out_stride=NOUT, workspace=r.ws[1].data_ptr(),
                      workspace_bytes=r.ws[1].numel(), stream=s)


bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
val = lambda t: M.from_bits(bits(t), M.BF16)


def against_the_plain_form(c, r):
    """The eager results within the bounds of the operators' own tests."""
    un, of = units.cpu().numpy(), off.cpu().numpy()
    lens, plen = c.lens.tolist(), int(c.groups[2][0])
    request, token = M.positions(np.concatenate([[0], np.cumsum(ROWS)]), lens)
    planes, past = ([p.cpu().numpy().reshape(total, chunk) for p in ps] for ps in (r.planes, c.past))
    new = [val(c.k), val(c.v)]

    def page(plane):                                    # [units, heads, page, dim] in 64 bits
        raw = np.ascontiguousarray(plane[:, :body])
        v = M.from_bits(raw if size == 1 else raw.view(np.uint16), kind).reshape(total, H, PAGE, D)
        if size == 1:
            s = np.ascontiguousarray(plane[:, body:]).view(np.float32).reshape(total, H, PAGE)
            v = v * s[..., None].astype(np.float64)
        return v

    kv = [page(p) for p in past]
    for i in range(2):
        held = M.stored(new[i], kind)
        for t in range(T):
            u, slot = un[of[request[t]] + token[t] // PAGE], token[t] % PAGE
            kv[i][u, :, slot] = held[t]
        assert np.array_equal(page(planes[i]), kv[i]), "planes"
        for t in range(T):
            u, slot = un[of[request[t]] + token[t] // PAGE], token[t] % PAGE
            w = kv[i][u, :, slot]
            assert (np.abs(val(r.back[i])[t] - w) <= np.abs(w) * (2.0 ** -8 + 2.0 ** -24)).all(), "back"
    of_agent = lambda i, a, n: np.concatenate([kv[i][un[of[a] + j]].transpose(1, 0, 2)
                                               for j in range(-(-n // PAGE))])[:n]
    out, lse, q, at = val(r.out), r.lse.cpu().numpy(), val(c.q), 0
    for a, n in enumerate(ROWS):
        if not n:
            continue
        L, P = lens[a], plen if a < R - 2 else 0
        k, v = (np.concatenate([of_agent(i, R, P), of_agent(i, a, L)]) if P else of_agent(i, a, L)
                for i in range(2))
        seen = np.arange(P + L) <= (P + L - n + np.arange(n))[:, None]
        o, l, mag, _, big = M.attention(q[at:at + n].reshape(n, H, PER, D), k, v, seen, D ** -0.5)
        e = ((D + 4) * 2.0 ** -24 * big + 2.0 ** -21)[..., None]
        tol = (2.0 ** -8 + 4 * e + (P + L + 64) * 2.0 ** -24) * mag + 2.0 ** -8 * np.abs(o)
        assert (np.abs(out[at:at + n].reshape(o.shape) - o) <= tol).all(), "attention"
        ltol = 2 * e[..., 0] + (P + L + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(l)
        assert (np.abs(lse[at:at + n].reshape(l.shape) - l) <= ltol).all(), "lse"
        u = un[of[a] + 3]
        want, second, first = M.adapter(val(c.x)[at:at + n], val(c.a[u]), val(c.b[u]), val(c.base)[at:at + n], 1.0)
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -16 + (2 * RANK + 8) * 2.0 ** -24) * second + \
            (NIN + 40) * 2.0 ** -24 * first + 2.0 ** -23 * np.abs(val(c.base)[at:at + n])
        assert (np.abs(val(r.y)[at:at + n] - want) <= tol).all(), "adapter"
        at += n


def same(r, want, what):
    for i, (x, y) in enumerate(zip(r.results(), want)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (what, i)


steps = [Step(), Step()]
runs = [[Run(c) for _ in range(RUNS)] for c in steps]


def eager(c, r):
    r.clear(c)
    c.call(r)
    torch.cuda.synchronize()
    return r.results()


for c, rs in zip(steps, runs):
    c.new()
    eager(c, rs[0])
    against_the_plain_form(c, rs[0])
print("plain ok", flush=True)
graphs = []
for c, rs in zip(steps, runs):
    for r in rs[:2]:                                    # two graphs of a step, workspaces apart
        r.clear(c)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.call(r)
        graphs.append((graph, c, r))
for turn in range(4):
    want = {}
    for c, rs in zip(steps, runs):
        c.new()
        want[c] = eager(c, rs[2])                       # outputs that no graph writes
    for graph, c, r in graphs if turn % 2 else graphs[::-1]:
        for again in range(2):
            r.clear(c)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            same(r, want[c], ("replay", turn, again))
    print("replays", turn, flush=True)
streams = [torch.cuda.Stream() for _ in range(2)]
for turn in range(3):
    want = []
    for c, rs in zip(steps, runs):
        c.new()
        want.append(eager(c, rs[0]))
        if turn == 0:
            against_the_plain_form(c, rs[0])
        for r in rs:
            r.clear(c)
    torch.cuda.synchronize()
    for i in range(RUNS):
        for c, rs, s in zip(steps, runs, streams):
            with torch.cuda.stream(s):
                c.call(rs[i])
    torch.cuda.synchronize()
    for rs, w in zip(runs, want):
        for i, r in enumerate(rs):
            same(r, w, ("streams", turn, i))
    # both streams replay graphs at once
    for graph, c, r in graphs:
        r.clear(c)
    torch.cuda.synchronize()
    for graph, c, r in graphs:
        with torch.cuda.stream(streams[steps.index(c)]):
            graph.replay()
    torch.cuda.synchronize()
    for graph, c, r in graphs:
        same(r, want[steps.index(c)], ("graphs on streams", turn))
    print("streams", turn, flush=True)
print("CHILD OK", flush=True)
'''


@pytest.mark.parametrize("rows", ["decode", "ragged"])
@pytest.mark.parametrize("kind", [B.SS_BF16, B.SS_E4M3])
def test_replays_and_streams(kind, rows):
    pytest.importorskip("torch")
    env = dict(os.environ, PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-u", "-c", CHILD, str(kind), rows], env=env, cwd=ROOT,
                       capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "CHILD OK" in r.stdout, r.stdout[-1500:] + r.stderr[-2500:]
