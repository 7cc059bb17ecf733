"""Measured operators: what a model that is served out of a memory pool does
with the units that the pool keeps resident.

Four operators over a pool's block table (``paper_2601_21473_amd.binding``):

``write``    the keys and values of new tokens go into their agents' pages, in
             16 bits as they are or as e4m3 with a scale per token and head;
``read``     tokens come back out of the pages, as 16-bit rows;
``attend``   attention of a ragged batch over the pages, where groups of
             requests share a prefix that is read once for all of them;
``adapter``  each request's own low-rank adapter, added to the output of the
             projection that all requests share.

A pool's plane is ``[units][chunk bytes]``.  A chunk holds a page of tokens,
head after head or token after token; in e4m3 the float scales follow the
codes as ``[heads][page]``.  Tokens of an agent are found through the block
table: its page j is unit ``units[agent_off[agent] + j]``, -1 where the agent
is not resident.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3_MAX = 448.0
SMALLEST = 2.0 ** -126      # a scale is at least this, so that it is never 0


def listed():
    return [
        # A decoding step's new tokens: 64 agents, one token each, 8 heads of
        # 128; a call is its launch.
        dict(name="write_decode", kind="write", requests=64, rows_lo=1, rows_hi=1, len_lo=200,
             len_hi=800, heads=8, dim=128, page=16, order="head", type="bf16", cache="e4m3", absent=0),
        # The prompts of 32 agents enter the cache: ragged, up to 1,000 tokens.
        dict(name="write_prompts", kind="write", requests=32, rows_lo=100, rows_hi=1000, len_lo=0,
             len_hi=300, heads=8, dim=128, page=16, order="head", type="bf16", cache="e4m3", absent=0),
        # Six agents of a small model (2 heads of 64, fp16, 256 tokens) read back.
        dict(name="read_small", kind="read", requests=6, rows_lo=256, rows_hi=256, len_lo=0, len_hi=0,
             heads=2, dim=64, page=16, order="token", type="f16", cache="f16", absent=0),
        # Prefixes of 64 agents (512 tokens, 8 heads of 128) out of an e4m3 cache.
        dict(name="read_prefixes", kind="read", requests=64, rows_lo=512, rows_hi=512, len_lo=0,
             len_hi=0, heads=8, dim=128, page=16, order="token", type="bf16", cache="e4m3", absent=0),
        # The smallest step: 6 active agents of the small model, 256 tokens
        # each, nothing shared.
        dict(name="attend_small", kind="attend", requests=6, groups=0, prefix_lo=0, prefix_hi=0,
             rows_lo=1, rows_hi=1, len_lo=256, len_hi=256, heads=2, per=2, dim=64, page=16,
             order="token", type="f16", cache="f16", absent=0),
        # One simulation: 64 agents that decode over the same world description
        # of 8,192 tokens, each with its own history.
        dict(name="attend_world", kind="attend", requests=64, groups=1, prefix_lo=8192,
             prefix_hi=8192, rows_lo=1, rows_hi=1, len_lo=100, len_hi=900, heads=8, per=4, dim=128,
             page=16, order="head", type="bf16", cache="bf16", absent=0),
        # Eight simulations side by side, 32 agents each, odd lengths, e4m3 cache.
        dict(name="attend_worlds_e4m3", kind="attend", requests=256, groups=8, prefix_lo=3001,
             prefix_hi=5003, rows_lo=1, rows_hi=1, len_lo=30, len_hi=1500, heads=8, per=4, dim=128,
             page=16, order="head", type="bf16", cache="e4m3", absent=0),
        # One agent with a very long history: split over the whole card, joined after.
        dict(name="attend_long", kind="attend", requests=1, groups=0, prefix_lo=0, prefix_hi=0,
             rows_lo=1, rows_hi=1, len_lo=131071, len_hi=131071, heads=8, per=4, dim=128, page=16,
             order="token", type="bf16", cache="bf16", absent=0),
        # Sixteen agents' prompts of about 500 tokens are computed over a shared
        # prefix: a matrix-product's worth of work.
        dict(name="attend_prompts", kind="attend", requests=16, groups=1, prefix_lo=4096,
             prefix_hi=4096, rows_lo=400, rows_hi=600, len_lo=0, len_hi=0, heads=8, per=4, dim=128,
             page=16, order="head", type="bf16", cache="bf16", absent=0),
        # 16 active agents, an adapter of rank 16 each, a square projection.
        dict(name="adapter_few", kind="adapter", requests=16, rows_lo=1, rows_hi=1, slots=64,
             rank=16, n_in=4096, n_out=4096, type="bf16", absent=0),
        # 256 decoding agents with skewed popularity over 200 adapters, a wide projection.
        dict(name="adapter_crowd", kind="adapter", requests=256, rows_lo=1, rows_hi=1, slots=200,
             rank=16, n_in=4096, n_out=14336, type="bf16", absent=0.02),
        # Prompts of 8 agents through rank-64 adapters of a smaller model, fp16.
        dict(name="adapter_prompts", kind="adapter", requests=8, rows_lo=300, rows_hi=700, slots=16,
             rank=64, n_in=2048, n_out=8192, type="f16", absent=0),
    ]


def _between(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "attend", "attend", "attend", "adapter", "adapter"])
    dim = rng.choice([64, 128, 128, 80, 256, 48])
    heads = rng.choice([1, 2, 4, 8])
    page = rng.choice([16, 16, 32, 64, 4, 1])
    order = rng.choice(["head", "token"])
    kt = rng.choice(["bf16", "f16"])
    cache = rng.choice([kt, "e4m3"])
    absent = rng.choice([0, 0, 0.1])
    if kind in ("write", "read"):
        rows = _between(rng, 1, 30_000)
        requests = min(rows, _between(rng, 1, 300))
        hi = max(1, rows // requests)
        rows_lo = rng.randint(1, hi)
        len_hi = rng.choice([0, rng.randint(1, 500)]) if kind == "write" else 0
        return dict(kind=kind, requests=requests, rows_lo=rows_lo, rows_hi=hi, len_lo=len_hi // 3,
                    len_hi=len_hi, heads=heads, dim=min(dim, 128) if rows > 8000 else dim, page=page,
                    order=order, type=kt, cache=cache, absent=absent)
    if kind == "attend":
        per = rng.choice([1, 2, 4, 8])
        shape = rng.choice(["decode", "decode", "short", "prompt"])
        if shape == "prompt":
            requests, rows_hi = rng.randint(1, 12), rng.randint(100, 500)
            groups = rng.choice([0, 1])
            prefix = _between(rng, 30, 3000)
            len_hi = 0
        else:
            requests = _between(rng, 1, 200)
            rows_hi = 1 if shape == "decode" else rng.randint(2, 9)
            groups = rng.choice([0, 1, 1, 4])
            groups = groups if requests >= groups else 1
            requests = requests // groups * groups if groups else requests
            prefix = _between(rng, 30, 9000)
            len_hi = _between(rng, 1, 100_000 // requests)
        return dict(kind=kind, requests=requests, groups=groups, prefix_lo=max(1, prefix * 2 // 3),
                    prefix_hi=prefix, rows_lo=1 if rng.random() < 0.5 else rows_hi, rows_hi=rows_hi,
                    len_lo=len_hi // 3, len_hi=len_hi, heads=heads, per=per, dim=dim, page=page,
                    order=order, type=kt, cache=cache, absent=absent)
    shape = rng.choice(["decode", "decode", "prompt"])
    requests = _between(rng, 1, 256) if shape == "decode" else rng.randint(1, 8)
    rows_hi = rng.choice([1, 1, 3]) if shape == "decode" else rng.randint(20, 700)
    n_in, n_out = (8 * _between(rng, 8, 600) for _ in range(2))
    return dict(kind=kind, requests=requests, rows_lo=1 if shape == "decode" else rows_hi // 2,
                rows_hi=rows_hi, slots=rng.randint(1, 200), rank=rng.choice([8, 16, 16, 32, 64, 128]),
                n_in=n_in, n_out=n_out, type=kt, absent=absent)


# ---- inputs -------------------------------------------------------------------


class State:
    """A case's inputs and what a program keeps between calls."""


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _sizes(case):
    """Lengths are the case's own, so that another seed's outputs have the same shapes."""
    return _generator(case["requests"] + 1000 * case["rows_hi"])


def _ints(lo, hi, n, g):
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int64)


def _offsets(counts):
    return torch.cat([counts.new_zeros(1), counts.cumsum(0)])


def _table(s, pages, absent, g):
    """A block table: each agent's pages at units in no order, some agents away."""
    s.agent_off = _offsets(pages)
    total = int(s.agent_off[-1])
    s.capacity = total + 7
    s.units = torch.randperm(s.capacity, generator=g, device="cuda")[:total].to(torch.int32)
    if absent:
        away = torch.rand(len(pages), generator=g, device="cuda") < absent
        s.units[torch.repeat_interleave(away, pages)] = -1


def _cache_views(s, plane):
    """A plane's codes or values [units, heads, page, dim] and, in e4m3, its
    scales [units, heads, page], as views of the plane's bytes."""
    kind = torch.float8_e4m3fn if s.quantised else s.dtype
    size = 1 if s.quantised else 2
    body = plane[:, :s.body].view(kind)
    stride = (s.chunk // size, s.head_bytes // size, s.token_bytes // size, 1)
    values = body.as_strided((s.capacity, s.heads, s.page, s.dim), stride)
    scales = plane.view(torch.float32).as_strided((s.capacity, s.heads, s.page),
                                                  (s.chunk // 4, s.page, 1),
                                                  s.body // 4) if s.quantised else None
    return values, scales


def _cache(s, case, g):
    """The key and value planes of one layer, filled with a past's contents."""
    s.heads, s.dim, s.page = case["heads"], case["dim"], case["page"]
    s.quantised = case["cache"] == "e4m3"
    size = 1 if s.quantised else 2
    if case["order"] == "head":
        s.token_bytes, s.head_bytes = s.dim * size, s.page * s.dim * size
    else:
        s.token_bytes, s.head_bytes = s.heads * s.dim * size, s.dim * size
    s.body = s.page * s.heads * s.dim * size
    s.chunk = -(-(s.body + (s.page * s.heads * 4 if s.quantised else 0)) // 16) * 16
    s.planes, s.views = [], []
    for _ in range(2):
        plane = torch.zeros((s.capacity, s.chunk), dtype=torch.uint8, device="cuda")
        values, scales = _cache_views(s, plane)
        past = torch.randn(values.shape, generator=g, device="cuda", dtype=torch.float32)
        if s.quantised:
            scale = past.abs().amax(-1).div_(E4M3_MAX).clamp_(min=SMALLEST)
            values.copy_((past / scale[..., None]).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn))
            scales.copy_(scale)
        else:
            values.copy_(past)
        s.planes.append(plane)
        s.views.append((values, scales))


def _rows(s, case):
    """Ragged requests: rows[r] rows each, of agents in no order."""
    n = case["requests"]
    s.rows = _ints(case["rows_lo"], case["rows_hi"], n, _sizes(case))
    s.row_off = _offsets(s.rows)
    s.n_rows = int(s.row_off[-1])
    s.most = int(s.rows.max())
    s.request = torch.repeat_interleave(torch.arange(n, device="cuda"), s.rows)
    s.place = torch.arange(s.n_rows, device="cuda") - s.row_off[s.request]


def prepare(case, seed):
    g = _generator(seed)
    s = State()
    s.kind, s.calls, s.requests = case["kind"], None, case["requests"]
    s.dtype = DTYPES[case["type"]]
    _rows(s, case)
    if case["kind"] == "adapter":
        s.rank, s.n_in, s.n_out = case["rank"], case["n_in"], case["n_out"]
        slots = case["slots"]
        _table(s, torch.ones(slots, dtype=torch.int64, device="cuda"), case["absent"], g)
        # popularity falls with the slot's number; 0.9 keeps more than one
        u = torch.rand(s.requests, generator=g, device="cuda")
        s.agents = (slots * u.pow(1.5)).long().clamp_(max=slots - 1)
        s.a = (torch.randn((s.capacity, s.rank, s.n_in), generator=g, device="cuda")
               / math.sqrt(s.n_in)).to(s.dtype)
        s.b = (torch.randn((s.capacity, s.n_out, s.rank), generator=g, device="cuda")
               / math.sqrt(s.rank)).to(s.dtype)
        s.x = torch.randn((s.n_rows, s.n_in), generator=g, device="cuda").to(s.dtype)
        s.base = torch.randn((s.n_rows, s.n_out), generator=g, device="cuda").to(s.dtype)
        s.out = torch.empty_like(s.base)
        s.scales = torch.rand(s.requests, generator=g, device="cuda") + 0.5
        s.slots = slots
    else:
        sizes = _sizes(case)
        past = _ints(case["len_lo"], case["len_hi"], s.requests, sizes)
        # a step's rows are the last of an agent's tokens; where there is only
        # one row, len is the whole history
        s.lens = torch.maximum(past, s.rows) if s.kind == "attend" else past + s.rows
        groups = case.get("groups", 0)
        s.prefix_lens = _ints(case["prefix_lo"], case["prefix_hi"], groups, sizes) if groups else \
            torch.zeros(0, dtype=torch.int64, device="cuda")
        s.groups = groups
        lens = torch.cat([s.lens, s.prefix_lens])
        spare = torch.ones(3, dtype=torch.int64, device="cuda")
        # agents in no order, three of them not in the batch
        order = torch.randperm(len(lens) + 3, generator=g, device="cuda")
        tokens = torch.cat([lens, spare])
        by_agent = torch.empty_like(tokens)
        by_agent[order] = tokens
        _table(s, (by_agent + case["page"] - 1) // case["page"], case["absent"], g)
        s.agents, s.prefix_agents = order[:s.requests], order[s.requests:s.requests + groups]
        s.n_agents = len(tokens)
        _cache(s, case, g)
        if groups:
            s.group_off = torch.arange(groups + 1, device="cuda") * (s.requests // groups)
        if s.kind == "attend":
            s.per = case["per"]
            s.q = torch.randn((s.n_rows, s.heads * s.per, s.dim), generator=g,
                              device="cuda").to(s.dtype)
            s.scale = 1 / math.sqrt(s.dim)
            s.out = torch.empty_like(s.q)
            s.lse = torch.empty((s.n_rows, s.heads * s.per), device="cuda")
        elif s.kind == "write":
            s.new = [torch.randn((s.n_rows, s.heads, s.dim), generator=g, device="cuda").to(s.dtype)
                     for _ in range(2)]
        else:
            s.got = [torch.empty((s.n_rows, s.heads, s.dim), dtype=s.dtype, device="cuda")
                     for _ in range(2)]
    # what the calls take: 32-bit indices, 64-bit table offsets
    s.row_off32, s.agents32 = s.row_off.to(torch.int32), s.agents.to(torch.int32)
    for name in ("lens", "prefix_lens", "prefix_agents", "group_off"):
        if hasattr(s, name):
            setattr(s, name + "32", getattr(s, name).to(torch.int32))
    torch.cuda.synchronize()
    return s


# ---- plain forms --------------------------------------------------------------


def _pages_of(s, agents, pages):
    """Units [len(agents), pages] of agents' first pages; -1 where there is none."""
    first = s.agent_off[agents][:, None] + torch.arange(pages, device="cuda")
    there = first < s.agent_off[agents + 1][:, None]
    return torch.where(there, s.units[first.clamp(max=len(s.units) - 1)].long(), -1)


def _tokens(s, view, agents, most):
    """Values [len(agents), heads, tokens, dim] of agents' first `most` tokens in
    32 bits, 0 where a page is away, and where there are tokens."""
    values, scales = view
    units = _pages_of(s, agents, max(1, -(-most // s.page)))
    there = units >= 0
    at = units.clamp(min=0)
    x = values[at].float()
    if scales is not None:
        x = x * scales[at][..., None]
    x = torch.where(there[:, :, None, None, None], x, 0.0)
    n, pages = units.shape
    x = x.permute(0, 2, 1, 3, 4).reshape(n, s.heads, pages * s.page, s.dim)
    return x, there.repeat_interleave(s.page, dim=1)


def _slots(s):
    """Unit and token-in-page of each row of the batch, and which rows have one."""
    position = s.lens[s.request] - s.rows[s.request] + s.place
    agent = s.agents[s.request]
    at = s.agent_off[agent] + position // s.page
    there = (position >= 0) & (at < s.agent_off[agent + 1])
    unit = s.units[at.clamp(0, len(s.units) - 1)].long()
    return unit, position % s.page, there & (unit >= 0)


def _write(s):
    unit, slot, there = _slots(s)
    unit, slot = unit[there], slot[there]
    out = []
    for new, (values, scales) in zip(s.new, s.views):
        x = new[there].float()
        if scales is None:
            values[unit, :, slot] = x.to(values.dtype)
            out.append(values)
        else:
            scale = (x.abs().amax(-1) / E4M3_MAX).clamp(min=SMALLEST)
            code = (x / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX)
            values.view(torch.uint8)[unit, :, slot] = code.to(torch.float8_e4m3fn).view(torch.uint8)
            scales[unit, :, slot] = scale
            out += [values, scales]
    return out


def _read(s):
    unit, slot, there = _slots(s)
    unit = unit.clamp(min=0)
    out = []
    for values, scales in s.views:
        if scales is None:
            x = values[unit, :, slot].float()
        else:
            x = values.view(torch.uint8)[unit, :, slot].view(torch.float8_e4m3fn).float()
            x = x * scales[unit, :, slot][..., None]
        out.append(torch.where(there[:, None, None], x, 0.0).to(s.dtype))
    return out


def _scores(s, q, k, seen):
    """Scaled scores of q [n, heads, rows, dim] with k [n, heads, keys, dim]."""
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) * s.scale
    return score.masked_fill_(~seen[:, None], -math.inf)


def _attend(s):
    n, h, per, most = s.requests, s.heads, s.per, s.most
    q = torch.zeros((n, most, h, per, s.dim), device="cuda")
    q[s.request, s.place] = s.q.float().view(s.n_rows, h, per, s.dim)
    q = q.permute(0, 2, 1, 3, 4).reshape(n, h, most * per, s.dim)
    row = torch.arange(most, device="cuda").repeat_interleave(per)
    # own tokens: row i sees own tokens 0 .. len - rows + i
    last = (s.lens - s.rows)[:, None] + row
    k, there = _tokens(s, s.views[0], s.agents, int(s.lens.max()))
    v, _ = _tokens(s, s.views[1], s.agents, int(s.lens.max()))
    seen = (torch.arange(k.shape[2], device="cuda") <= last[:, :, None]) & there[:, None]
    own_score = _scores(s, q, k, seen)
    top = own_score.amax(-1)
    if s.groups:
        # the prefix once for all requests of its group
        each = n // s.groups
        longest = int(s.prefix_lens.max())
        pk, pthere = _tokens(s, s.views[0], s.prefix_agents, longest)
        pv, _ = _tokens(s, s.views[1], s.prefix_agents, longest)
        key = torch.arange(pk.shape[2], device="cuda")
        plen = s.prefix_lens.repeat_interleave(each)
        bound = torch.minimum(plen[:, None], plen[:, None] + last + 1).view(s.groups, -1)
        pseen = (key < bound[:, :, None]) & pthere[:, None]
        stack = q.view(s.groups, each, h, most * per, s.dim).transpose(1, 2).reshape(
            s.groups, h, each * most * per, s.dim)
        score = _scores(s, stack, pk, pseen)

        def apart(x):
            return x.view(s.groups, h, each, most * per, -1).transpose(1, 2).reshape(
                n, h, most * per, -1)

        top = torch.maximum(top, apart(score.amax(-1))[..., 0])
    base = torch.where(torch.isinf(top), 0.0, top)
    weight = torch.exp(own_score - base[..., None])
    total = weight.sum(-1)
    out = torch.matmul(weight, v)
    if s.groups:
        spread = base.view(s.groups, each, h, most * per).transpose(1, 2).reshape(
            s.groups, h, each * most * per)
        weight = torch.exp(score - spread[..., None])
        total = total + apart(weight.sum(-1))[..., 0]
        out = out + apart(torch.matmul(weight, pv))
    lse = torch.where(total > 0, base + total.log(), -math.inf)
    out = out / torch.where(total > 0, total, 1.0)[..., None]

    def rows(x):
        x = x.view(n, h, most, per, -1).permute(0, 2, 1, 3, 4)[s.request, s.place]
        return x.reshape(s.n_rows, h * per, -1)

    return rows(out).to(s.dtype), rows(lse)[..., 0]


def _adapter(s):
    unit = s.units[s.agent_off[s.agents]].long()
    scale = torch.where(unit >= 0, s.scales, 0.0)
    unit = unit.clamp(min=0)
    x = torch.zeros((s.requests, s.most, s.n_in), device="cuda")
    x[s.request, s.place] = s.x.float()
    low = torch.matmul(x, s.a[unit].float().transpose(1, 2).contiguous())
    add = torch.matmul(low, s.b[unit].float().transpose(1, 2).contiguous())
    add = add * scale[:, None, None]
    return (s.base.float() + add[s.request, s.place]).to(s.dtype)


# ---- the framework's calls ----------------------------------------------------


def _calls(s, ss):
    """The descriptors and the workspace that a program makes once."""
    t = {torch.bfloat16: ss.SS_BF16, torch.float16: ss.SS_F16}[s.dtype]
    if s.kind == "adapter":
        size = s.a.element_size()
        handle = ss.adapters(units=s.units.data_ptr(), agent_off=s.agent_off.data_ptr(),
                             n_agents=s.slots, n_entries=len(s.units), capacity_units=s.capacity,
                             a=s.a.data_ptr(), b=s.b.data_ptr(),
                             a_unit_bytes=s.rank * s.n_in * size,
                             b_unit_bytes=s.rank * s.n_out * size, rank=s.rank, n_in=s.n_in,
                             n_out=s.n_out, type=t)
        batch = ss.batch(n_rows=s.n_rows, n_requests=s.requests, row_off=s.row_off32.data_ptr(),
                         agents=s.agents32.data_ptr())
        need = ss.adapter_add_workspace(handle, s.n_rows, s.requests)
    else:
        handle = ss.kv_cache(units=s.units.data_ptr(), agent_off=s.agent_off.data_ptr(),
                             n_agents=s.n_agents, n_entries=len(s.units), capacity_units=s.capacity,
                             k=s.planes[0].data_ptr(), v=s.planes[1].data_ptr(),
                             k_unit_bytes=s.chunk, v_unit_bytes=s.chunk, page_tokens=s.page,
                             n_heads=s.heads, head_dim=s.dim,
                             type=ss.SS_E4M3 if s.quantised else t, token_bytes=s.token_bytes,
                             head_bytes=s.head_bytes, scale_off=s.body if s.quantised else 0)
        groups = dict(n_groups=s.groups, group_off=s.group_off32.data_ptr(),
                      prefix_agents=s.prefix_agents32.data_ptr(),
                      prefix_lens=s.prefix_lens32.data_ptr()) if s.groups else {}
        batch = ss.batch(n_rows=s.n_rows, n_requests=s.requests, row_off=s.row_off32.data_ptr(),
                         agents=s.agents32.data_ptr(), lens=s.lens32.data_ptr(), **groups)
        need = ss.prefix_attention_workspace(handle, batch, s.heads * s.per) \
            if s.kind == "attend" else 0
    return t, handle, batch, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")


def _run_own(s):
    from paper_2601_21473_amd import binding as ss
    if s.calls is None:
        s.calls = _calls(s, ss)
    t, handle, batch, work = s.calls
    stream = torch.cuda.current_stream().cuda_stream
    if s.kind == "adapter":
        ss.adapter_add(handle, batch, x=s.x.data_ptr(), base=s.base.data_ptr(), out=s.out.data_ptr(),
                       x_stride=s.n_in, base_stride=s.n_out, out_stride=s.n_out,
                       scales=s.scales.data_ptr(), workspace=work.data_ptr(),
                       workspace_bytes=work.numel(), stream=stream)
        return s.out
    if s.kind == "attend":
        strides = (s.heads * s.per * s.dim, s.dim)
        ss.prefix_attention(handle, batch, q=s.q.data_ptr(), out=s.out.data_ptr(),
                            lse=s.lse.data_ptr(), type=t, n_q_heads=s.heads * s.per,
                            q_strides=strides, out_strides=strides, scale=s.scale,
                            workspace=work.data_ptr(), workspace_bytes=work.numel(), stream=stream)
        return s.out, s.lse
    strides = (s.heads * s.dim, s.dim)
    if s.kind == "write":
        ss.kv_write(handle, batch, k=s.new[0].data_ptr(), v=s.new[1].data_ptr(), type=t,
                    strides=strides, stream=stream)
        return [x for view in s.views for x in view if x is not None]
    ss.kv_read(handle, batch, k=s.got[0].data_ptr(), v=s.got[1].data_ptr(), type=t, strides=strides,
               stream=stream)
    return s.got


def run(state):
    if own:
        return _run_own(state)
    return {"write": _write, "read": _read, "attend": _attend, "adapter": _adapter}[state.kind](state)


# ---- what a pass cannot do without ----------------------------------------------


def work(case):
    mean_rows = (case["rows_lo"] + case["rows_hi"]) / 2
    rows = case["requests"] * mean_rows
    if case["kind"] == "adapter":
        rank, n_in, n_out = case["rank"], case["n_in"], case["n_out"]
        used = case["slots"] * (1 - (1 - 1 / case["slots"]) ** case["requests"])
        return {"bytes": 2 * (rows * (n_in + 2 * n_out) + used * rank * (n_in + n_out)),
                "flops": 2 * rows * rank * (n_in + n_out)}
    heads, dim = case["heads"], case["dim"]
    token = dim + 4 if case["cache"] == "e4m3" else 2 * dim
    if case["kind"] != "attend":
        return {"bytes": 2 * rows * heads * (2 * dim + token), "flops": 2 * rows * heads * dim}
    mean_len = max((case["len_lo"] + case["len_hi"]) / 2, mean_rows)
    prefix = (case["prefix_lo"] + case["prefix_hi"]) / 2 if case["groups"] else 0
    keys = prefix + mean_len - (mean_rows - 1) / 2
    cached = case["groups"] * prefix + case["requests"] * mean_len
    q_heads = heads * case["per"]
    return {"bytes": 2 * heads * cached * token + rows * q_heads * (4 * dim + 4),
            "flops": 4 * rows * q_heads * dim * keys}


# ---- from the definition, in 64 bits --------------------------------------------


def _row_of(s, agent, token):
    """The unit and slot of one agent's tokens (host lists of the table)."""
    j = token // s.page
    first, last = s.off_host[agent], s.off_host[agent + 1]
    return int(s.units_host[first + j]) if 0 <= j < last - first else -1, token % s.page


def _stored(s, view, agent, count):
    """An agent's first tokens [count, heads, dim] in 64 bits and which are there."""
    pages = -(-count // s.page)
    units = [_row_of(s, agent, j * s.page)[0] for j in range(pages)]
    there = torch.tensor([u >= 0 for u in units], device="cuda").repeat_interleave(s.page)[:count]
    at = torch.tensor([max(u, 0) for u in units], device="cuda")
    values = view[0].view(torch.uint8 if s.quantised else view[0].dtype)[at].transpose(1, 2)
    values = values.reshape(pages * s.page, s.heads, -1)[:count].contiguous()
    x = values.view(torch.float8_e4m3fn).to(torch.float64) if s.quantised else values.double()
    if s.quantised:
        x = x * view[1][at].transpose(1, 2).reshape(pages * s.page, s.heads)[:count, :, None].double()
    x[~there] = 0
    return x, there


def exact(case, seed):
    s = prepare(case, seed)
    s.off_host, s.units_host = s.agent_off.tolist(), s.units.tolist()
    rows, agents, start = s.rows.tolist(), s.agents.tolist(), s.row_off.tolist()
    if s.kind == "adapter":
        out = s.base.double()
        for r in range(s.requests):
            unit = s.units_host[s.off_host[agents[r]]]
            if unit >= 0:
                at = slice(start[r], start[r] + rows[r])
                low = s.x[at].double() @ s.a[unit].double().T
                out[at] += s.scales[r].double() * (low @ s.b[unit].double().T)
        return out
    lens = s.lens.tolist()
    if s.kind == "write":
        # the quotients before their rounding to 8 bits
        out = []
        for new, view in zip(s.new, s.views):
            values = view[0].to(torch.float64)
            scales = view[1].double() if s.quantised else None
            at, unit, slot = [], [], []
            for r in range(s.requests):
                for i in range(rows[r]):
                    u, t = _row_of(s, agents[r], lens[r] - rows[r] + i)
                    if u >= 0:
                        at.append(start[r] + i)
                        unit.append(u)
                        slot.append(t)
            at, unit, slot = (torch.tensor(x, dtype=torch.int64, device="cuda")
                              for x in (at, unit, slot))
            x = new.double()[at]
            if s.quantised:
                scale = (x.abs().amax(-1) / E4M3_MAX).clamp(min=SMALLEST)
                x = x / scale[..., None]
                scales[unit, :, slot] = scale
            values[unit, :, slot] = x
            out += [values] if scales is None else [values, scales]
        return out
    if s.kind == "read":
        return [torch.cat([_stored(s, view, agents[r], lens[r])[0][lens[r] - rows[r]:]
                           for r in range(s.requests)]) for view in s.views]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s.lse.shape, -math.inf, dtype=torch.float64, device="cuda")
    shared = [[_stored(s, view, a, n) for view in s.views]
              for a, n in zip(s.prefix_agents.tolist(), s.prefix_lens.tolist())] if s.groups else []
    for r in range(s.requests):
        (k, there), (v, _) = (_stored(s, view, agents[r], lens[r]) for view in s.views)
        before = 0
        if s.groups:
            (pk, pthere), (pv, _) = shared[r // (s.requests // s.groups)]
            before = len(pk)
            k, v, there = torch.cat([pk, k]), torch.cat([pv, v]), torch.cat([pthere, there])
        at = slice(start[r], start[r] + rows[r])
        q = s.q[at].double().view(rows[r], s.heads, s.per, s.dim).permute(1, 2, 0, 3)
        position = before + lens[r] - rows[r] + torch.arange(rows[r], device="cuda")
        seen = (torch.arange(len(k), device="cuda") <= position[:, None]) & there
        for h in range(s.heads):
            score = (q[h] @ k[:, h].T.contiguous()) * s.scale
            score = score.masked_fill(~seen, -math.inf)
            total = torch.logsumexp(score, -1)
            weight = torch.exp(score - torch.where(torch.isinf(total), 0.0, total)[..., None])
            out.view(s.n_rows, s.heads, s.per, s.dim)[at, h] = (weight @ v[:, h].contiguous()
                                                                ).transpose(0, 1)
            lse.view(s.n_rows, s.heads, s.per)[at, h] = total.T
    return out, lse
