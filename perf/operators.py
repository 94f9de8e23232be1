"""Operators behind answering with a model: what a program calls between the linears of a layer when it continues
sequences out of a paged cache of keys and values.

Kinds of call:
  plan     block tables and slots of the tokens that the running sequences add, blocks taken from and given back to a
           list of free ones: qzo_cache_plan
  rotate   heads of q and k normed (RMSNorm over a head) and rotated to their positions, k and v written into the cache
           at their slots, or without a cache q and k of a batch of sequences: qzo_qk_norm_rope
  attend   attention of the newest tokens over the cache, through the block tables: qzo_paged_attention

A case is a dict of plain values; `prepare` makes what such a program holds before the call, `run` is one call, `work`
the bytes and operations that it cannot do without, `exact` the result from the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
NORM_EPS = 1e-6


def listed():
    return [
        # eight sequences being continued by a token each: nothing but latency
        dict(name="plan_8_tokens", kind="plan", n_seq=8, short=17, long=4000, added=1, ended=0, block=16),
        # a thousand of them, some of which have just ended
        dict(name="plan_1000_tokens", kind="plan", n_seq=1000, short=1, long=8000, added=1, ended=37, block=32),
        # prompts coming in beside sequences that go on
        dict(name="plan_300_prompts", kind="plan", n_seq=300, short=0, long=3000, added=801, ended=5, block=64),
        # one token of one sequence, heads of the 7B shape, rotation and cache
        dict(name="rotate_1_token", kind="rotate", tokens=1, q_heads=32, kv_heads=32, dh=128, norm=False, cache="bf16", block=16, far=4096),
        # prompts of the 13B shape into the cache, heads normed
        dict(name="rotate_2500_tokens", kind="rotate", tokens=2500, q_heads=40, kv_heads=40, dh=128, norm=True, cache="bf16", block=32,
             far=131072),
        # shared key heads of 64, an 8-bit cache
        dict(name="rotate_e4m3_7001_tokens", kind="rotate", tokens=7001, q_heads=64, kv_heads=8, dh=64, norm=True, cache="e4m3", block=64,
             far=32768),
        # the batch of a training step at the 7B shape, 16 sequences of 512: q and k of whole sequences, no cache
        dict(name="rotate_16x512", kind="rotate", tokens=8192, q_heads=32, kv_heads=32, dh=128, norm=True, cache="none", block=16, far=512),
        # a single sequence of the 7B shape's longest: few keys, latency
        dict(name="attend_1x512", kind="attend", n_seq=1, short=512, long=512, empty=0, new=1, q_heads=32, kv_heads=32, dh=128,
             cache="bf16", block=16),
        # a batch of sequences of all lengths, a key head for every query head
        dict(name="attend_64_ragged", kind="attend", n_seq=64, short=19, long=4001, empty=1, new=1, q_heads=32, kv_heads=32, dh=128,
             cache="bf16", block=32),
        # a few very long sequences, shared key heads
        dict(name="attend_8x65536", kind="attend", n_seq=8, short=65536, long=65536, empty=0, new=1, q_heads=64, kv_heads=8, dh=128,
             cache="bf16", block=64),
        # the same in 8 bits, ragged
        dict(name="attend_e4m3_24_ragged", kind="attend", n_seq=24, short=700, long=32001, empty=0, new=1, q_heads=40, kv_heads=8, dh=128,
             cache="e4m3", block=32),
        # pieces of prompts behind what is cached already, heads of 64
        dict(name="attend_6x100_new", kind="attend", n_seq=6, short=300, long=2222, empty=0, new=100, q_heads=32, kv_heads=32, dh=64,
             cache="bf16", block=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["plan", "rotate", "rotate", "attend", "attend", "attend"])
    block = rng.choice([16, 32, 64, 128])
    if kind == "plan":
        n_seq, added = _log_int(rng, 1, 1500), rng.choice([1, 1, _log_int(rng, 2, 900)])
        long = _log_int(rng, 2, 8000)
        return dict(kind=kind, n_seq=n_seq if added == 1 else min(n_seq, max(1, 240000 // added)), short=min(long, rng.choice([0, 1, 33])), long=long,
                    added=added, ended=rng.choice([0, n_seq // 50]) if added == 1 else 0, block=block)
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8, 16])
    while kv_heads * group > 128:
        group //= 2
    dh = rng.choice([64, 128, 128])
    heads = dict(q_heads=kv_heads * group, kv_heads=kv_heads, dh=dh)
    if kind == "rotate":
        cache = rng.choice(["bf16", "bf16", "e4m3", "none"])
        most = 8192 * 64 * 128 // ((heads["q_heads"] + 2 * kv_heads) * dh)
        return dict(kind=kind, tokens=min(_log_int(rng, 1, 8192), most), **heads, norm=rng.random() < 0.6, cache=cache, block=block,
                    far=rng.choice([512, 4096, 32768, 131072]))
    # at most some 2^19 positions of eight key heads of 128
    n_seq = _log_int(rng, 1, 256)
    most = (1 << 29) // (n_seq * kv_heads * dh)
    long = max(1, min(_log_int(rng, 1, 65536), most))
    new = rng.choice([1, 1, 1, 1, _log_int(rng, 2, 120)])
    if new > 1:
        long = max(new, min(long, (1 << 28) // (n_seq * heads["q_heads"] * new)))
        if n_seq * long * kv_heads * dh > 1 << 29:
            new, long = 1, most
    return dict(kind=kind, n_seq=n_seq, short=max(new, int(long * rng.choice([1.0, 0.3, 0.02]))), long=long, empty=rng.choice([0, 0, 1]) if new == 1 else 0,
                new=new, **heads, cache=rng.choice(["bf16", "bf16", "e4m3"]), block=block)


def _lengths(case):
    """Lengths of the sequences: spread over [short, long] by their logarithm; the order of the list is prepare's."""
    n, lo, hi = case["n_seq"], case["short"], case["long"]
    got = [int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** (i / max(1, n - 1)))) - 1 for i in range(n)]
    got[-1] = hi
    for i in range(case.get("empty", 0)):
        if n > 1:
            got[i] = 0
    return got


def _blocks(tokens, block):
    return -(-tokens // block)


def _prepare_plan(case, gen):
    n, block = case["n_seq"], case["block"]
    order = torch.randperm(n, generator=gen)
    cached = torch.tensor(_lengths(case), dtype=torch.int32)[order]
    added = torch.full((n,), case["added"], dtype=torch.int32)
    if case["added"] > 1:       # every third sequence goes on by a token
        added[torch.arange(n) % 3 == 1] = 1
    max_tokens = int(added.sum()) + 5          # a batch padded by a few rows
    ended = torch.randperm(n, generator=gen)[:case["ended"]]
    added[ended] = -1
    old = (cached + block - 1) // block
    max_blocks = _blocks(case["long"] + case["added"], block) + 1
    used = int(old.sum())
    n_blocks = used + _blocks(max_tokens, block) + n + 8
    ids = torch.randperm(n_blocks, generator=gen).to(torch.int32)
    tables = torch.full((n, max_blocks), -1, dtype=torch.int32)
    held = torch.arange(max_blocks)[None, :] < old[:, None]
    tables[held] = ids[:used]
    free = torch.full((n_blocks,), -1, dtype=torch.int32)
    free[:n_blocks - used] = ids[used:]
    state = torch.tensor([n_blocks - used, 0, 0, 0], dtype=torch.int32)
    st = dict(cached=cached, added=added, tables=tables, free=free, state=state)
    st = {k: v.to(DEV) for k, v in st.items()}
    st.update(block=block, lengths=torch.zeros(n, dtype=torch.int32, device=DEV), starts=torch.zeros(n + 1, dtype=torch.int32, device=DEV),
              slots=torch.zeros(max_tokens, dtype=torch.int32, device=DEV), positions=torch.zeros(max_tokens, dtype=torch.int32, device=DEV),
              after=torch.zeros(4, dtype=torch.int32, device=DEV))
    return st


def _run_plan(st):
    cached, added, tables, free, block = st["cached"], st["added"], st["tables"], st["free"], st["block"]
    n, max_blocks = tables.shape
    n_blocks, max_tokens, n_free = free.numel(), st["slots"].numel(), st["state"][0]
    zero = torch.zeros_like(cached)
    ended = added < 0
    after = torch.where(ended, zero, cached + added)
    old, new = (cached + block - 1) // block, (after + block - 1) // block
    back = torch.where(ended, old, zero).cumsum(0)               # blocks given back, sequence by sequence
    take = torch.where(ended, zero, new - old).cumsum(0)
    starts = torch.nn.functional.pad(added.clamp(min=0).cumsum(0), (1, 0))
    n_back, n_take, n_tokens = back[-1], take[-1], starts[-1]
    # blocks given back lie on top of the free ones, in order; taken ones come off the top
    k = torch.arange(n_blocks, device=DEV)
    giver = torch.searchsorted(back, k, right=True).clamp(max=n - 1)
    given = tables[giver, (k - back[giver] + old[giver]).clamp(0, max_blocks - 1)]
    stack = torch.where(k < n_free, free, given[(k - n_free).clamp(0, n_blocks - 1)])
    taken = stack[(n_free + n_back - 1 - k).clamp(0, n_blocks - 1)]
    taker = torch.searchsorted(take, k, right=True).clamp(max=n - 1)
    place = taker * max_blocks + old[taker] + k - (take[taker] - (new - old)[taker])
    wide = torch.cat([tables.reshape(-1), zero[:1]])             # one place more, for what is not taken
    wide[torch.where(k < n_take, place, n * max_blocks)] = taken
    tables.copy_(wide[:-1].view(n, max_blocks))
    left = n_free + n_back - n_take
    free.copy_(torch.where((k >= n_free) & (k < left), stack, free))
    t = torch.arange(max_tokens, device=DEV)
    seq = torch.searchsorted(starts, t, right=True).sub(1).clamp(max=n - 1)
    at = cached[seq] + t - starts[seq]
    slot = tables[seq, (at // block).clamp(0, max_blocks - 1)] * block + at % block
    some = t < n_tokens
    st["lengths"].copy_(after)
    st["starts"].copy_(starts)
    st["slots"].copy_(torch.where(some, slot, -1))
    st["positions"].copy_(torch.where(some, at, 0))
    st["after"].copy_(torch.stack([left, n_tokens, torch.zeros_like(left), n_take]))
    return [tables, free, st["lengths"], st["starts"], st["slots"], st["positions"], st["after"]]


def _prepare_cache(case, n_blocks, gen, filled):
    shape = (n_blocks, case["kv_heads"], case["block"], case["dh"])
    k, v = ((torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16) if filled else torch.zeros(shape, device=DEV, dtype=torch.bfloat16))
            for _ in range(2))
    scale = [None, None]
    if case["cache"] == "e4m3":
        # values of magnitude 1 stored as up to some 30 steps of the scale
        scale = [torch.rand(case["kv_heads"], generator=gen, device=DEV) * 0.1 + 0.05 for _ in range(2)]
        if filled:
            k, v = (torch.cat([(p.float() * 8).to(torch.float8_e4m3fn) for p in x.split(max(1, (1 << 26) // x[0].numel()))]) for x in (k, v))
        else:
            k, v = (x.to(torch.float8_e4m3fn) for x in (k, v))
    return dict(k=k, v=v, k_scale=scale[0], v_scale=scale[1])


def _prepare_rotate(case, gen):
    T, H, Hk, dh = case["tokens"], case["q_heads"], case["kv_heads"], case["dh"]
    st = dict(q_heads=H, kv_heads=Hk, theta=10000.0, q_gain=None, k_gain=None, slots=None, cache=None)
    # rows of a projection, heads of different size
    x = torch.randn(T, H + 2 * Hk, dh, generator=gen, device=DEV) * (torch.rand(1, H + 2 * Hk, 1, generator=gen, device=DEV) * 2 + 0.3)
    st["qkv"] = x.to(torch.bfloat16).view(T, -1)
    if case["norm"]:
        st["q_gain"], st["k_gain"] = ((1 + 0.2 * torch.randn(dh, generator=gen, device=DEV)).to(torch.bfloat16) for _ in range(2))
    if case["cache"] == "none":
        st["out"] = torch.zeros(T, (H + Hk) * dh, dtype=torch.bfloat16, device=DEV)
        st["positions"] = torch.arange(T, device=DEV, dtype=torch.int32) % case["far"]
        return st
    st["out"] = torch.zeros(T, H * dh, dtype=torch.bfloat16, device=DEV)
    st["positions"] = (torch.arange(T, device=DEV, dtype=torch.int32) * 7 + torch.randint(0, case["far"], (1,), generator=gen, device=DEV,
                                                                                         dtype=torch.int32)) % case["far"]
    n_blocks = _blocks(T, case["block"]) + 1
    st["slots"] = torch.randperm(n_blocks * case["block"], generator=gen, device=DEV)[:T].to(torch.int32)
    st["cache"] = _prepare_cache(case, n_blocks, gen, False)
    return st


def _store(pool, slots, x, scale):
    """Rows x [T, kv_heads, dh] to their slots of a pool [blocks, kv_heads, block, dh]."""
    block, at = pool.shape[2], slots.long()
    if pool.dtype == torch.float8_e4m3fn:
        x = x if scale is None else x / scale[:, None]
        x = x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        pool.view(torch.uint8)[at // block, :, at % block] = x
    else:
        pool[at // block, :, at % block] = x.to(pool.dtype)


def _run_rotate(st):
    T, H, Hk = st["qkv"].shape[0], st["q_heads"], st["kv_heads"]
    x = st["qkv"].view(T, H + 2 * Hk, -1).float()
    q, k, v = x[:, :H], x[:, H:H + Hk], x[:, H + Hk:]
    dh = q.shape[-1]
    if st["q_gain"] is not None:
        q = q * (q.square().mean(-1, keepdim=True) + NORM_EPS).rsqrt() * st["q_gain"].float()
        k = k * (k.square().mean(-1, keepdim=True) + NORM_EPS).rsqrt() * st["k_gain"].float()
    # angles of far positions: in 64 bits
    angle = st["positions"].double()[:, None] * st["theta"] ** (-torch.arange(dh // 2, device=DEV, dtype=torch.float64) * 2 / dh)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(a):
        lo, hi = a[..., :dh // 2], a[..., dh // 2:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)

    q, k = turned(q), turned(k)
    if st["cache"] is None:
        st["out"].copy_(torch.cat([q, k], 1).reshape(T, -1))
        return [st["out"]]
    c = st["cache"]
    st["out"].copy_(q.reshape(T, -1))
    _store(c["k"], st["slots"], k, c["k_scale"])
    _store(c["v"], st["slots"], v, c["v_scale"])
    return [st["out"], c["k"], c["v"]]


def _prepare_attend(case, gen, cpu):
    n, block, new, H, dh = case["n_seq"], case["block"], case["new"], case["q_heads"], case["dh"]
    lens = torch.tensor(_lengths(case))[torch.randperm(n, generator=cpu)]
    need = (lens + block - 1) // block
    used, max_blocks = int(need.sum()), max(1, int(need.max()))
    n_blocks = used + 3
    tables = torch.full((n, max_blocks), -1, dtype=torch.int32)
    tables[torch.arange(max_blocks)[None, :] < need[:, None]] = torch.randperm(n_blocks, generator=cpu)[:used].to(torch.int32)
    st = dict(cache=_prepare_cache(case, n_blocks, gen, True), tables=tables.to(DEV), lengths=lens.to(torch.int32).to(DEV), new=new, q_heads=H, dh=dh,
              scale=1.0 / math.sqrt(dh))
    # scores of a standard deviation of 2.5: some keys stand out
    st["q"] = (torch.randn(n * new, H * dh, generator=gen, device=DEV) * 2.5).to(torch.bfloat16)
    st["starts"] = torch.arange(n + 1, device=DEV, dtype=torch.int32) * new if new > 1 else None
    st["out"] = torch.zeros(n * new, H * dh, dtype=torch.bfloat16, device=DEV)
    return st


def _gathered(pool, tables, scale):
    """Keys or values of every sequence behind one another, fp32 [n_seq, kv_heads, positions, dh]."""
    n, kv_heads, dh = tables.shape[0], pool.shape[1], pool.shape[3]
    x = pool.view(torch.uint8)[tables.long().clamp(min=0)].view(pool.dtype) if pool.dtype == torch.float8_e4m3fn else pool[tables.long().clamp(min=0)]
    x = x.transpose(1, 2).float().reshape(n, kv_heads, -1, dh)
    return x if scale is None else x * scale[:, None, None]


def _run_attend(st):
    c, lens, new = st["cache"], st["lengths"].long(), st["new"]
    n, kv_heads, dh = st["tables"].shape[0], c["k"].shape[1], st["dh"]
    group = st["q_heads"] // kv_heads
    k = _gathered(c["k"], st["tables"], c["k_scale"])
    # columns: the heads that share a key head, token by token
    q = st["q"].view(n, new, kv_heads, group, dh).float().permute(0, 2, 4, 1, 3).reshape(n, kv_heads, dh, new * group).contiguous()
    s = torch.matmul(k, q) * st["scale"]
    del k
    sees = (lens[:, None] - new + 1 + torch.arange(new, device=DEV)).clamp(min=0).repeat_interleave(group, 1)       # [n, new * group]
    mask = torch.arange(s.shape[2], device=DEV)[None, :, None] < sees[:, None, :]
    s = s.masked_fill(~mask[:, None], -math.inf)
    p = (s - s.amax(2, keepdim=True).clamp(min=-1e30)).exp()
    p = (p / p.sum(2, keepdim=True).clamp(min=1e-30)).transpose(2, 3).contiguous()
    o = torch.matmul(p, _gathered(c["v"], st["tables"], c["v_scale"]))
    st["out"].copy_(o.view(n, kv_heads, new, group, dh).transpose(1, 2).reshape(n * new, -1))
    return [st["out"]]


def prepare(case, seed):
    gen, cpu = torch.Generator(device=DEV), torch.Generator()
    gen.manual_seed(seed)
    cpu.manual_seed(seed)
    kind = case["kind"]
    st = _prepare_plan(case, cpu) if kind == "plan" else _prepare_rotate(case, gen) if kind == "rotate" else _prepare_attend(case, gen, cpu)
    st["kind"] = kind
    return st


def _run_own(st):
    from paper_2505_13430_amd import binding as qb
    if st["kind"] == "plan":
        qb.qzo_cache_plan(st["cached"], st["added"], st["block"], st["tables"], st["free"], st["state"], st["lengths"], st["starts"], st["slots"],
                          st["positions"], st["after"])
        return [st["tables"], st["free"], st["lengths"], st["starts"], st["slots"], st["positions"], st["after"]]
    c = st["cache"]
    cache = None if c is None else qb.make_cache(c["k"], c["v"], c["k_scale"], c["v_scale"])
    if st["kind"] == "rotate":
        qb.qzo_qk_norm_rope(st["qkv"], st["q_heads"], st["kv_heads"], st["out"], q_gain=st["q_gain"], k_gain=st["k_gain"], eps=NORM_EPS,
                            theta=st["theta"], positions=st["positions"], cache=cache, slots=st["slots"])
        return [st["out"]] if c is None else [st["out"], c["k"], c["v"]]
    qb.qzo_paged_attention(st["q"], cache, st["tables"], st["lengths"], st["out"], st["scale"], starts=st["starts"])
    return [st["out"]]


def run(state):
    if own:
        return _run_own(state)
    kind = state["kind"]
    return _run_plan(state) if kind == "plan" else _run_rotate(state) if kind == "rotate" else _run_attend(state)


def work(case):
    if case["kind"] == "plan":
        n, block, lens = case["n_seq"], case["block"], _lengths(case)
        tokens = n * case["added"] if case["added"] == 1 else n * (2 * case["added"] + 1) // 3
        blocks = tokens // block
        # lengths and counts in, lengths and starts out; a slot and a position of every token; taken blocks read and entered
        return {"bytes": 4.0 * (4 * n + 2 * tokens + 2 * blocks) + (4.0 * sum(lens) / block / max(1, n) * case["ended"] if case["ended"] else 0.0),
                "flops": 0.0}
    H, Hk, dh = case["q_heads"], case["kv_heads"], case["dh"]
    wide = 1 if case["cache"] == "e4m3" else 2
    if case["kind"] == "rotate":
        T = case["tokens"]
        if case["cache"] == "none":
            return {"bytes": 4.0 * T * (H + Hk) * dh + 4.0 * T, "flops": 10.0 * T * (H + Hk) * dh}
        return {"bytes": T * (2.0 * (H + 2 * Hk) * dh + 2.0 * H * dh + 2.0 * Hk * dh * wide + 8.0), "flops": 10.0 * T * (H + Hk) * dh}
    lens, new = _lengths(case), case["new"]
    keys = sum(lens)
    pairs = sum(new * max(0, length) - new * (new - 1) // 2 if length >= new else 0 for length in lens)
    return {"bytes": 2.0 * keys * Hk * dh * wide + 4.0 * case["n_seq"] * new * H * dh + 4.0 * keys / case["block"], "flops": 4.0 * pairs * H * dh}


def _exact_head(x, gain):
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + NORM_EPS) * gain.double()


def _exact_rotate(case, st):
    T, H, Hk, dh = case["tokens"], case["q_heads"], case["kv_heads"], case["dh"]
    heads = st["qkv"].double().view(T, H + 2 * Hk, dh)
    q, k, v = heads.split([H, Hk, Hk], 1)
    if case["norm"]:
        q, k = _exact_head(q, st["q_gain"]), _exact_head(k, st["k_gain"])
    i = torch.arange(dh // 2, device=DEV, dtype=torch.float64)
    turn = torch.polar(torch.ones(T, 1, dh // 2, device=DEV, dtype=torch.float64),
                       (st["positions"].double()[:, None] * torch.exp(-2.0 * i / dh * math.log(st["theta"]))[None])[:, None])
    q, k = (torch.view_as_real(torch.complex(x[..., :dh // 2], x[..., dh // 2:]) * turn) for x in (q.contiguous(), k.contiguous()))
    q, k = (torch.cat([x[..., 0], x[..., 1]], -1) for x in (q, k))
    if case["cache"] == "none":
        return [torch.cat([q, k], 1).reshape(T, -1)]
    got = [q.reshape(T, -1)]
    for x, name in ((k, "k"), (v, "v")):
        if st["cache"][name + "_scale"] is not None:
            x = x / st["cache"][name + "_scale"].double()[None, :, None]
        flat = torch.zeros(st["cache"][name].shape[0] * case["block"], Hk, dh, device=DEV, dtype=torch.float64)
        flat[st["slots"].long()] = x
        got.append(flat.view(-1, case["block"], Hk, dh).transpose(1, 2).contiguous())
    return got


def _exact_attend(case, st):
    n, new, block, Hk, dh = case["n_seq"], case["new"], case["block"], case["kv_heads"], case["dh"]
    group, out = case["q_heads"] // Hk, []
    pools = []
    for name in ("k", "v"):
        scale = st["cache"][name + "_scale"]
        pools.append((st["cache"][name], torch.ones(Hk, device=DEV) if scale is None else scale))
    q = st["q"].double().view(n, new, Hk, group, dh)
    for b in range(n):
        length = int(st["lengths"][b])
        if length == 0:
            out.append(torch.zeros(new, Hk * group * dh, device=DEV, dtype=torch.float64))
            continue
        at = torch.arange(length, device=DEV)
        ids = st["tables"][b].long()[at // block]
        rows = []
        for h in range(Hk):
            k, v = (pool[:, h].contiguous().view(torch.uint8).view(-1, dh * pool.element_size())[ids * block + at % block].view(pool.dtype).double() * scale[h].double()
                    for pool, scale in pools)
            s = torch.mm(q[b, :, h].reshape(new * group, dh), k.t().contiguous()) * st["scale"]
            late = at[None, :] > (length - new + torch.arange(new, device=DEV)).repeat_interleave(group)[:, None]
            rows.append(torch.mm(torch.softmax(s.masked_fill(late, -math.inf), -1), v).view(new, 1, group * dh))
        out.append(torch.cat(rows, 1).reshape(new, -1))
    return [torch.cat(out)]


def exact(case, seed):
    if case["kind"] == "plan":
        return None                       # whole numbers, no rounding
    if case["kind"] == "attend" and case["n_seq"] * case["kv_heads"] > 4096:
        return None                       # thousands of small products
    st = prepare(case, seed)
    return _exact_rotate(case, st) if case["kind"] == "rotate" else _exact_attend(case, st)
