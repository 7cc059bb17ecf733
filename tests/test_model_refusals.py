"""What the operators over resident units refuse, before any device work (CPU)."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2601_21473_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x100000                                        # an aligned address that is no memory


def cache(**kw):
    a = dict(units=P, agent_off=P, n_agents=4, n_entries=8, capacity_units=8, k=P, v=P,
             k_unit_bytes=16384, v_unit_bytes=16384, page_tokens=16, n_heads=2, head_dim=64,
             type=B.SS_BF16, token_bytes=128, head_bytes=2048, scale_off=0)
    a.update(kw)
    return B.kv_cache(**a)


def batch(**kw):
    a = dict(n_rows=4, n_requests=2, row_off=P, agents=P, lens=P)
    a.update(kw)
    return B.batch(**a)


def adapters(**kw):
    a = dict(units=P, agent_off=P, n_agents=4, n_entries=4, capacity_units=8, a=P, b=P,
             a_unit_bytes=4096, b_unit_bytes=4096, rank=16, n_in=64, n_out=64, type=B.SS_F16)
    a.update(kw)
    return B.adapters(**a)


def refused(msg, call, *args, **kw):
    with pytest.raises(B.ScaleSimError, match=msg) as e:
        call(*args, **kw)
    assert e.value.status == B.SS_ERR_ARG


def write(c=None, b=None, **kw):
    a = dict(k=P, v=P, type=B.SS_BF16, strides=(128, 64))
    a.update(kw)
    k, v = a.pop("k"), a.pop("v")
    B.kv_write(c or cache(), b or batch(), k, v, **a)
    B.kv_read(c or cache(), b or batch(), k, v, **a)


def attend(c=None, b=None, **kw):
    a = dict(q=P, out=2 * P, type=B.SS_BF16, n_q_heads=4, q_strides=(256, 64), out_strides=(256, 64),
             scale=1.0, workspace=4 * P, workspace_bytes=1 << 30)
    a.update(kw)
    B.prefix_attention(c or cache(), b or batch(), a.pop("q"), a.pop("out"), **a)


def add(d=None, b=None, **kw):
    a = dict(x=P, base=2 * P, out=2 * P, x_stride=64, base_stride=64, out_stride=64, workspace=4 * P,
             workspace_bytes=1 << 20)
    a.update(kw)
    B.adapter_add(d or adapters(), b or batch(lens=0), a.pop("x"), a.pop("base"), a.pop("out"), **a)


CACHES = [
    (dict(units=0), "NULL block table"), (dict(agent_off=0), "NULL block table"),
    (dict(n_agents=0), "n_agents"), (dict(n_entries=0), "n_entries"),
    (dict(capacity_units=0), "capacity_units"), (dict(capacity_units=1 << 31), "capacity_units"),
    (dict(k=0), "aligned"), (dict(v=P + 8), "aligned"), (dict(page_tokens=0), "page_tokens"),
    (dict(page_tokens=24), "page_tokens"), (dict(page_tokens=2048), "page_tokens"),
    (dict(n_heads=0), "n_heads"), (dict(n_heads=1025), "n_heads"), (dict(head_dim=0), "head_dim"),
    (dict(head_dim=72), "head_dim"), (dict(head_dim=272), "head_dim"), (dict(type=0), "unknown cache type"),
    (dict(type=4), "unknown cache type"), (dict(type=B.SS_F16), "with a cache of type"),
    (dict(token_bytes=136), "multiples of 16"), (dict(k_unit_bytes=16392), "multiples of 16"),
    (dict(token_bytes=112), "overlap"), (dict(head_bytes=1024), "overlap"),
    (dict(head_bytes=2032), "overlap"), (dict(token_bytes=128, head_bytes=128), "overlap"),
    (dict(v_unit_bytes=4080), "does not fit"),
    (dict(type=B.SS_E4M3, token_bytes=64, head_bytes=1024, scale_off=2032), "inside the page"),
    (dict(type=B.SS_E4M3, token_bytes=64, head_bytes=1024, scale_off=16384), "does not fit"),
    (dict(k_unit_bytes=1 << 62), "too large"), (dict(token_bytes=1 << 63, head_bytes=128), "does not fit|large"),
    (dict(capacity_units=1, token_bytes=1 << 28, head_bytes=128), "too large"),
]


@pytest.mark.parametrize("change,msg", CACHES)
def test_caches(change, msg):
    refused(msg, write, cache(**change))
    refused(msg, attend, cache(**change))


BATCHES = [(dict(n_rows=1 << 31), "n_rows"), (dict(n_requests=1 << 20), "n_requests"),
           (dict(row_off=0), "NULL array"), (dict(agents=0), "NULL array")]


@pytest.mark.parametrize("change,msg", BATCHES)
def test_batches(change, msg):
    refused(msg, write, None, batch(**change))
    refused(msg, attend, None, batch(**change))
    refused(msg, add, None, batch(**change))


def test_lens_and_groups():
    refused("NULL array", write, None, batch(lens=0))
    refused("NULL array", attend, None, batch(lens=0))
    refused("groups", attend, None, batch(n_groups=1))
    refused("n_groups", attend, None, batch(n_groups=1 << 20))


@pytest.mark.parametrize("change,msg", [
    (dict(k=0), "k must be"), (dict(v=P + 2), "v must be"), (dict(strides=(130, 64)), "multiples of 8"),
    (dict(strides=(128, 60)), "multiples of 8"), (dict(type=B.SS_E4M3), "rows must be"),
    (dict(type=0), "rows must be"), (dict(strides=(1 << 41, 64)), "too large")])
def test_rows(change, msg):
    refused(msg, write, **change)


def test_rows_that_overlap_are_refused_where_they_are_written():
    a = dict(type=B.SS_BF16, strides=(64, 64))
    refused("overlap", B.kv_read, cache(), batch(), P, P, **a)
    refused("current device|device memory", B.kv_write, cache(), batch(), P, P, **a)


@pytest.mark.parametrize("change,msg", [
    (dict(q=0), "q must be"), (dict(out=8), "out must be"), (dict(n_q_heads=3), "n_q_heads"),
    (dict(n_q_heads=0), "n_q_heads"), (dict(n_q_heads=65538), "n_q_heads"),
    (dict(scale=float("nan")), "scale"), (dict(scale=3e38), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(out=P), "out overlaps q"), (dict(out=P + 1024), "out overlaps q"),
    (dict(out_strides=(64, 64)), "overlap"), (dict(q_strides=(4, 64)), "multiples of 8"),
    (dict(workspace=0), "workspace"), (dict(workspace=P + 4), "workspace"),
    (dict(workspace_bytes=1000), "workspace_bytes"), (dict(type=B.SS_F16), "with a cache of type")])
def test_attention(change, msg):
    refused(msg, attend, **change)


def test_attention_of_too_many_rows():
    refused("2\\^30", attend, None, batch(n_rows=1 << 28))


@pytest.mark.parametrize("change,msg", [
    (dict(units=0), "NULL block table"), (dict(n_entries=0), "n_entries"), (dict(a=0), "aligned"),
    (dict(b=P + 4), "aligned"), (dict(rank=0), "rank"), (dict(rank=12), "rank"), (dict(rank=136), "rank"),
    (dict(n_in=0), "n_in"), (dict(n_in=60), "n_in"), (dict(n_out=1 << 24), "n_out"),
    (dict(type=B.SS_E4M3), "SS_BF16 or SS_F16"), (dict(a_unit_bytes=4104), "multiples of 16"),
    (dict(b_unit_bytes=1 << 31), "below 2"),
    (dict(rank=128, n_out=(1 << 24) - 8, capacity_units=1), "too large"), (dict(a_unit_bytes=1024), "does not fit")])
def test_adapters(change, msg):
    refused(msg, add, adapters(**change))
    assert B.adapter_add_workspace(adapters(**change), 4, 2) == 0


@pytest.mark.parametrize("change,msg", [
    (dict(x=0), "x must be"), (dict(base=8), "base must be"), (dict(out=0), "out must be"),
    (dict(x_stride=60), "multiples of 8"), (dict(out_stride=56), "overlap"),
    (dict(out=P), "out overlaps x"), (dict(out=2 * P + 128), "out overlaps base"),
    (dict(out_stride=128), "out overlaps base"), (dict(workspace=0), "workspace"),
    (dict(workspace_bytes=16), "workspace_bytes")])
def test_adapter_rows(change, msg):
    refused(msg, add, **change)


def test_memory_that_is_none():
    """Everything else in order: the pointers are not memory of a device."""
    for call in (write, attend, add):
        refused("current device|device memory", call)


def test_null_structs():
    L = B.load()
    b, c = batch(), cache()
    for st in (L.ss_kv_write(None, C.byref(b), P, P, 1, 128, 64, None),
               L.ss_kv_read(C.byref(c), None, P, P, 1, 128, 64, None),
               L.ss_prefix_attention(None, None, P, P, None, 1, 4, 256, 64, 256, 64, 1.0, P, 1, None),
               L.ss_adapter_add(None, C.byref(b), P, P, P, 64, 64, 64, None, P, 1, None)):
        assert st == B.SS_ERR_ARG
    assert L.ss_prefix_attention_workspace(None, None, 4) == 0
    assert L.ss_adapter_add_workspace(None, 4, 2) == 0


def test_nothing_to_do_is_fine():
    for change in (dict(n_rows=0), dict(n_requests=0)):
        b = batch(**change, row_off=0, agents=0, lens=0)
        write(None, b)
        attend(None, b)
        add(None, b)


def test_workspaces_grow_with_the_batch():
    small = B.prefix_attention_workspace(cache(), batch(), 4)
    assert 0 < small < B.prefix_attention_workspace(cache(), batch(n_rows=400), 4)
    assert B.prefix_attention_workspace(cache(), batch(), 3) == 0
    assert 0 < B.adapter_add_workspace(adapters(), 4, 2) < B.adapter_add_workspace(adapters(), 400, 2)


def test_struct_layouts_match_header(tmp_path):
    structs = {"ss_kv_cache": B.ss_kv_cache, "ss_batch": B.ss_batch, "ss_adapters": B.ss_adapters}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "scalesim.h"', "int main(void){"]
    for sname, cls in structs.items():
        lines.append(f'printf("{sname} size %zu\\n", sizeof({sname}));')
        for f, _ in cls._fields_:
            lines.append(f'printf("{sname}.{f} %zu\\n", offsetof({sname}, {f}));')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    got = dict(line.rsplit(" ", 1) for line in out.strip().splitlines())
    for sname, cls in structs.items():
        assert int(got[f"{sname} size"]) == C.sizeof(cls), sname
        for f, _ in cls._fields_:
            assert int(got[f"{sname}.{f}"]) == getattr(cls, f).offset, (sname, f)
    text = open(os.path.join(ROOT, "include", "scalesim.h")).read()
    for name in ("SS_BF16", "SS_F16", "SS_E4M3"):
        assert int(re.search(rf"#define {name}\s+(\d+)u", text).group(1)) == getattr(B, name)


def test_pool_helpers_check_the_chunks():
    """Pool.kv_cache and Pool.adapters, on a pool that was never created."""
    pool = B.Pool.__new__(B.Pool)
    pool._h, pool.n_agents, pool._capacity = None, 4, 8
    pool._units = np.ones(4, np.uint32)
    pool._chunk = np.array([4096, 4096, 4224], np.uint64)
    pool._bases = [P, 2 * P, 3 * P]
    pool.block_table = lambda: (P, P)
    kw = dict(page_tokens=16, n_heads=2, head_dim=64)
    c = pool.kv_cache(0, 1, type=B.SS_BF16, **kw)
    assert (c.k, c.v, c.k_unit_bytes, c.token_bytes, c.head_bytes) == (P, 2 * P, 4096, 128, 2048)
    assert (c.n_entries, c.capacity_units, c.n_agents) == (4, 8, 4)
    c = pool.kv_cache(2, 0, type=B.SS_E4M3, order="token", k_offset=1024, **kw)
    assert (c.k, c.token_bytes, c.head_bytes, c.scale_off) == (3 * P + 1024, 128, 64, 2048)
    with pytest.raises(ValueError, match="plane 1"):
        pool.kv_cache(0, 1, type=B.SS_BF16, v_offset=16, **kw)
    with pytest.raises(KeyError):
        pool.kv_cache(0, 1, type=B.SS_BF16, order="dim", **kw)
    a = pool.adapters(0, 2, rank=16, n_in=128, n_out=132, type=B.SS_F16, unit=1)
    assert (a.a, a.b, a.b_unit_bytes, a.unit) == (P, 3 * P, 4224, 1)
    with pytest.raises(ValueError, match="plane 0"):
        pool.adapters(0, 2, rank=16, n_in=136, n_out=128, type=B.SS_F16)
