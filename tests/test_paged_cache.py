"""The paged cache of keys and values: block tables and slots, heads of q and k into the cache, attention over it, against
plain implementations in 64 bits (whole numbers: equal).

Tolerances are what the roundings add up to.  eps/2 of bf16 is 2^-8, of e4m3 2^-4, of fp32 2^-24."""
import ctypes as C
import math
import threading

import numpy as np
import pytest
import torch

from paper_2505_13430_amd import binding as qb

DEV = "cuda:0"
gpu = pytest.mark.gpu


# ------------------------------------------------------------------ plain implementations ----
def plan_reference(cached, added, block, tables, free, n_free, max_tokens):
    """The stack of free blocks as a list; what a failing plan leaves is the caller's to compare."""
    n, most = tables.shape
    tables, lengths, starts, slots, positions = tables.copy(), [], [0], [], []
    stack = list(free[:n_free])
    held = [-(-c // block) for c in cached]
    if n_free < 0 or n_free > len(free) or min(cached) < 0:
        return qb.QZO_ERR_ARG
    if any(c + max(a, 0) > most * block for c, a in zip(cached, added)) or sum(max(a, 0) for a in added) > max_tokens:
        return qb.QZO_ERR_SHAPE
    for i in range(n):
        if added[i] < 0:
            stack += list(tables[i, :held[i]])
    if len(stack) > len(free):
        return qb.QZO_ERR_ARG
    had = len(stack)
    for i in range(n):
        length = 0 if added[i] < 0 else cached[i] + added[i]
        if added[i] >= 0:
            for j in range(held[i], -(-length // block)):
                if not stack:
                    return qb.QZO_ERR_WORKSPACE
                tables[i, j] = stack.pop()
            for p in range(cached[i], length):
                slots.append(tables[i, p // block] * block + p % block)
                positions.append(p)
        lengths.append(length)
        starts.append(len(slots))
    after = free.copy()
    after[n_free:len(stack)] = stack[n_free:]
    pad = max_tokens - len(slots)
    return dict(tables=tables, free=after, lengths=lengths, starts=starts, slots=slots + [-1] * pad, positions=positions + [0] * pad,
                after=[len(stack), starts[-1], 0, had - len(stack)])


def rope_reference(x, positions, theta):
    """x fp64 [T, heads, dh]; also the sum of the two products' magnitudes of every feature."""
    dh = x.shape[-1]
    if theta == 0:
        return x, x.abs()
    angle = positions.double()[:, None, None] * theta ** (-torch.arange(dh // 2, dtype=torch.float64) * 2 / dh)
    c, s = angle.cos(), angle.sin()
    lo, hi = x[..., :dh // 2], x[..., dh // 2:]
    return (torch.cat([lo * c - hi * s, hi * c + lo * s], -1),
            torch.cat([(lo * c).abs() + (hi * s).abs(), (hi * c).abs() + (lo * s).abs()], -1))


def norm_reference(x, gain, eps):
    return x if gain is None else x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * gain.double()


def attention_reference(q, k, v, tables, lengths, starts, scale):
    """q [rows, heads, dh], pools [n_blocks, kv_heads, block, dh], all fp64 on the host; starts a list.  Returns the output and
    sum p |v| / sum p, with the largest sum |q| |k| of a row's scores; None for rows that starts does not name."""
    group, block = q.shape[1] // k.shape[1], k.shape[2]
    out, mag, mac = torch.full_like(q, math.nan), torch.zeros_like(q), torch.zeros_like(q[..., 0])
    for i in range(len(lengths)):
        for r in range(starts[i], starts[i + 1]):
            sees = min(lengths[i], tables.shape[1] * block) - (starts[i + 1] - 1 - r)
            at = torch.arange(max(0, sees), device=q.device)
            ids = tables[i, at // block].long()
            at, ids = at[(ids >= 0) & (ids < k.shape[0])], ids[(ids >= 0) & (ids < k.shape[0])]
            if at.numel() == 0:
                out[r] = 0
                continue
            kk, vv = (p[ids, :, at % block].repeat_interleave(group, 1) for p in (k, v))         # [keys, heads, dh]
            s = scale * (q[r][None] * kk).sum(-1)
            p = torch.softmax(s, 0)
            out[r], mag[r] = (p[..., None] * vv).sum(0), (p[..., None] * vv.abs()).sum(0)
            mac[r] = (abs(scale) * (q[r].abs()[None] * kk.abs()).sum(-1)).amax(0)
    return out, mag, mac


def attention_tolerance(out, mag, mac, dh):
    """One rounding of the output, one of every p to bf16, before it meets v and the sum, both 2^-8: p_k (1 + e_k) in both gives
    out + sum p_k e_k (v_k - out) / sum p_k (1 + e_k), at most 2^-8 (sum p |v| / sum p + |out|) / (1 - 2^-8) away.  Scores in fp32: dh products
    and sums and two more factors, (dh + 4) 2^-24 of sum |q| |k| at most, that much of a p's logarithm and twice that of its share."""
    return 2.0 ** -8 * out.abs() + (2.0 ** -8 * (mag + out.abs()) + 2 * (dh + 4) * 2.0 ** -24 * mac[..., None] * mag) * 1.01 + 1e-30


# ------------------------------------------------------------------ refusals, on the host ----
def _p(address=16):
    return C.c_void_p(address)


def _cache(**over):
    v = dict(struct_size=C.sizeof(qb.qzo_cache), type=0, n_blocks=8, block=16, kv_heads=2, head_dim=64, k_dev=16, v_dev=16, k_scale_dev=None,
             v_scale_dev=None)
    v.update(over)
    return qb.qzo_cache(*v.values())


BAD_CACHES = [(dict(struct_size=4), qb.QZO_ERR_ARG), (dict(type=2), qb.QZO_ERR_UNSUPPORTED), (dict(k_dev=None), qb.QZO_ERR_ARG), (dict(v_dev=24), qb.QZO_ERR_ALIGN),
              (dict(k_scale_dev=16), qb.QZO_ERR_ARG), (dict(block=24), qb.QZO_ERR_SHAPE), (dict(block=8), qb.QZO_ERR_SHAPE), (dict(block=512), qb.QZO_ERR_SHAPE),
              (dict(head_dim=96), qb.QZO_ERR_SHAPE), (dict(n_blocks=0), qb.QZO_ERR_SHAPE), (dict(n_blocks=1 << 27), qb.QZO_ERR_SHAPE),
              (dict(kv_heads=0), qb.QZO_ERR_SHAPE)]


@pytest.mark.parametrize("over,status", [
    (dict(cached=None), qb.QZO_ERR_ARG), (dict(after=None), qb.QZO_ERR_ARG), (dict(slots=24), qb.QZO_ERR_ALIGN), (dict(n_seq=0), qb.QZO_ERR_SHAPE),
    (dict(n_seq=8193), qb.QZO_ERR_SHAPE), (dict(block=17), qb.QZO_ERR_SHAPE), (dict(n_blocks=0), qb.QZO_ERR_SHAPE), (dict(max_blocks=0), qb.QZO_ERR_SHAPE),
    (dict(n_seq=4096, max_blocks=1 << 19), qb.QZO_ERR_SHAPE), (dict(max_tokens=0), qb.QZO_ERR_SHAPE), (dict(max_tokens=1 << 31), qb.QZO_ERR_SHAPE)])
def test_plan_refuses(over, status):
    v = dict(cached=16, added=16, n_seq=2, block=16, n_blocks=8, max_blocks=4, max_tokens=8, tables=16, free=16, before=16, lengths=16, starts=16,
             slots=16, positions=16, after=16)
    v.update(over)
    assert qb.lib().qzo_cache_plan(*v.values(), None) == status and qb.lib().qzo_last_error()


@pytest.mark.parametrize("over,status", [
    (dict(qkv=None), qb.QZO_ERR_ARG), (dict(out=None), qb.QZO_ERR_ARG), (dict(slots=16), qb.QZO_ERR_ARG), (dict(out=24), qb.QZO_ERR_ALIGN),
    (dict(q_gain=20), qb.QZO_ERR_ALIGN), (dict(dh=96), qb.QZO_ERR_SHAPE), (dict(q_heads=0), qb.QZO_ERR_SHAPE), (dict(kv_heads=0), qb.QZO_ERR_SHAPE),
    (dict(eps=-1.0), qb.QZO_ERR_ARG), (dict(eps=math.nan), qb.QZO_ERR_ARG), (dict(theta=-1.0), qb.QZO_ERR_ARG), (dict(theta=math.inf), qb.QZO_ERR_ARG),
    (dict(seq=0), qb.QZO_ERR_ARG), (dict(ldx=508), qb.QZO_ERR_SHAPE), (dict(ldx=504), qb.QZO_ERR_SHAPE), (dict(ldy=376), qb.QZO_ERR_SHAPE),
    (dict(tokens=1 << 25), qb.QZO_ERR_SHAPE), (dict(out=16, ldx=512, ldy=384), qb.QZO_ERR_ARG)])
def test_qk_norm_rope_refuses(over, status):
    v = dict(qkv=16, ldx=512, tokens=4, q_heads=4, kv_heads=2, dh=64, q_gain=None, k_gain=None, eps=1e-6, theta=10000.0, positions=None, seq=8, cache=None,
             slots=None, out=32, ldy=384)
    v.update(over)
    assert qb.lib().qzo_qk_norm_rope(*v.values(), None) == status and qb.lib().qzo_last_error()


@pytest.mark.parametrize("over,status", BAD_CACHES + [(dict(kv_heads=4), qb.QZO_ERR_SHAPE), (dict(head_dim=128), qb.QZO_ERR_SHAPE)])
def test_qk_norm_rope_refuses_caches(over, status):
    c = _cache(**over)
    assert qb.lib().qzo_qk_norm_rope(16, 512, 4, 4, 2, 64, None, None, 1e-6, 1e4, 16, 0, C.addressof(c), 16, 32, 256, None) == status


@pytest.mark.parametrize("over,status", [
    (dict(q=None), qb.QZO_ERR_ARG), (dict(cache=None), qb.QZO_ERR_ARG), (dict(tables=None), qb.QZO_ERR_ARG), (dict(lengths=20), qb.QZO_ERR_ALIGN),
    (dict(starts=20), qb.QZO_ERR_ALIGN), (dict(n_seq=0), qb.QZO_ERR_SHAPE), (dict(n_seq=8193), qb.QZO_ERR_SHAPE), (dict(q_heads=5), qb.QZO_ERR_SHAPE),
    (dict(q_heads=0), qb.QZO_ERR_SHAPE), (dict(max_blocks=0), qb.QZO_ERR_SHAPE), (dict(max_blocks=1 << 27), qb.QZO_ERR_SHAPE), (dict(max_blocks=(1 << 26) + 1), qb.QZO_ERR_SHAPE), (dict(ldq=252), qb.QZO_ERR_SHAPE),
    (dict(ldo=248), qb.QZO_ERR_SHAPE), (dict(scale=math.nan), qb.QZO_ERR_ARG), (dict(rows=1 << 30), qb.QZO_ERR_SHAPE)])
def test_paged_attention_refuses(over, status):
    c = _cache()
    v = dict(q=16, ldq=256, rows=2, n_seq=2, q_heads=4, cache=C.addressof(c), tables=16, max_blocks=4, lengths=16, starts=None, scale=0.125, out=16,
             ldo=256, scratch=256, bytes=1 << 40)
    v.update(over)
    assert qb.lib().qzo_paged_attention(*v.values(), None) == status and qb.lib().qzo_last_error()


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_paged_attention_refuses_caches(over, status):
    c = _cache(**over)
    assert qb.lib().qzo_paged_attention(16, 256, 2, 2, 4, C.addressof(c), 16, 4, 16, None, 0.125, 16, 256, 256, 1 << 40, None) == status


# ------------------------------------------------------------------ block tables and slots ----
def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def _plan(cached, added, block, tables, free, n_free, max_tokens, in_place=False):
    n = len(cached)
    d = dict(cached=_i32(cached), added=_i32(added), tables=_i32(tables), free=_i32(free), before=_i32([n_free, 7, 7, 7]),
             lengths=_i32([-5] * n), starts=_i32([-5] * (n + 1)), slots=_i32([-5] * max_tokens), positions=_i32([-5] * max_tokens),
             after=_i32([-5] * 4))
    if in_place:
        d["lengths"], d["after"] = d["cached"], d["before"]
    qb.qzo_cache_plan(d["cached"], d["added"], block, d["tables"], d["free"], d["before"], d["lengths"], d["starts"], d["slots"], d["positions"],
                      d["after"])
    return {k: d[k].cpu().numpy() for k in ("tables", "free", "lengths", "starts", "slots", "positions", "after")}


def _pool(cached, block, spare, most, seed):
    """Tables that hold the cached tokens, a shuffled free list of `spare` blocks, entries beyond either of -9."""
    rng = np.random.default_rng(seed)
    held = [-(-c // block) for c in cached]
    ids = rng.permutation(sum(held) + spare)
    tables, at = np.full((len(cached), most), -9), 0
    for i, h in enumerate(held):
        tables[i, :h] = ids[at:at + h]
        at += h
    free = np.full(len(ids), -9)
    free[:spare] = ids[at:]
    return tables, free


@gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cached,added,block", [
    ([0], [1], 16), ([15], [1], 16), ([16], [1], 16), ([5], [0], 32), ([40], [-1], 16), ([0, 0, 0], [0, -1, 0], 16),
    ([31, 32, 33, 0, 64], [1, 1, 1, 70, -1], 32), ([100, 7, 255, 256, 0, 9], [-1, 300, 1, 1, 0, -1], 256), ([17] * 5, [-1] * 5, 16)])
def test_plan(cached, added, block, in_place):
    tables, free = _pool(cached, block, 9, 1 + max(c + max(a, 0) for c, a in zip(cached, added)) // block + 1, 1)
    tokens = sum(max(a, 0) for a in added) + 3
    want = plan_reference(cached, added, block, tables, free, 9, tokens)
    got = _plan(cached, added, block, tables, free, 9, tokens, in_place)
    for k, v in want.items():
        assert np.array_equal(got[k], v), (k, got[k], v)


@gpu
@pytest.mark.parametrize("n,block,longest,most_added,ends,pad,seed", [
    (63, 16, 300, 5, 0.2, 1, 1), (1023, 16, 90, 1, 0.1, 100, 2), (1025, 32, 200, 9, 0.3, 1, 3), (3000, 64, 500, 2, 0.02, 9, 4),
    (8192, 16, 60, 3, 0.1, 1, 5), (8192, 16, 60, 0, 0.3, 4000, 8), (40, 128, 9000, 4000, 0.1, 77, 6), (2, 16, 10, 40000, 0.0, 1, 7)])
def test_plan_of_many(n, block, longest, most_added, ends, pad, seed):
    """From one to 8192 sequences, with more than 4096 tokens and fewer."""
    rng = np.random.default_rng(seed)
    cached, added = rng.integers(0, longest + 1, n), rng.integers(0, most_added + 1, n)
    added[rng.random(n) < ends] = -1
    added[0] = most_added
    tables, free = _pool(cached, block, n + int(added.clip(0).sum()) // block, (longest + most_added) // block + 1, seed)
    n_free, tokens = n + int(added.clip(0).sum()) // block, int(added.clip(0).sum()) + pad
    want = plan_reference(cached.tolist(), added.tolist(), block, tables, free, n_free, tokens)
    got = _plan(cached, added, block, tables, free, n_free, tokens, in_place=seed % 2 == 0)
    for k, v in want.items():
        assert np.array_equal(got[k], v), k


@gpu
@pytest.mark.parametrize("cached,added,n_free,most,tokens,status", [
    ([16, 16], [1, 1], 1, 4, 2, qb.QZO_ERR_WORKSPACE), ([16, 16], [17, 1], 2, 4, 20, qb.QZO_ERR_WORKSPACE), ([64, 3], [1, 1], 9, 4, 2, qb.QZO_ERR_SHAPE),
    ([65, 3], [-1, 1], 4, 4, 2, qb.QZO_ERR_SHAPE), ([5, 3], [2, 1], 9, 4, 2, qb.QZO_ERR_SHAPE), ([-1, 3], [1, 1], 9, 4, 2, qb.QZO_ERR_ARG),
    ([5, 3], [1, 1], -1, 4, 2, qb.QZO_ERR_ARG), ([5, 3], [1, 1], 99, 4, 2, qb.QZO_ERR_ARG), ([64, 64], [-1, -1], 6, 4, 2, qb.QZO_ERR_ARG),
    ([0, 0], [2 ** 31 - 1, 2 ** 31 - 1], 9, 4, 5000, qb.QZO_ERR_SHAPE)])
def test_plan_that_cannot_be_made_changes_nothing(cached, added, n_free, most, tokens, status):
    tables, free = np.arange(2 * most).reshape(2, most) % 9, np.arange(9)
    ref = plan_reference(cached, added, 16, tables, free, n_free, tokens)
    assert ref == status
    for in_place in (False, True):
        got = _plan(cached, added, 16, tables, free, n_free, tokens, in_place)
        assert np.array_equal(got["tables"], tables) and np.array_equal(got["free"], free) and got["lengths"].tolist() == cached
        assert not got["starts"].any() and (got["slots"] == -1).all() and not got["positions"].any()
        assert got["after"].tolist() == [n_free, 0, status, 0]


@gpu
@pytest.mark.parametrize("n,added,pad", [(6, 1, 2), (6, 40, 2), (1100, 1, 3), (1100, 5, 3), (6, 40, 4100)])
def test_plan_gives_no_slot_in_a_block_outside_the_pool(n, added, pad):
    """Ids that shifted by the block's size would wrap to another block's slots, in the tables and on the free list; tokens that a thread
    itself sees to, prompts, and more than 4096 of them."""
    block, cached = 16, [20 + i % 16 for i in range(n)]
    tables, free = _pool(cached, block, 4 * n, 6, 11)
    bad = [1 << 28, (1 << 28) + 1, -1, len(free), 2 ** 31 - 1, -2 ** 31]
    for i, x in enumerate(bad):
        tables[(3 * i + 1) % n, 1] = x
    free[4 * n - len(bad):4 * n] = bad
    tokens = n * added + pad
    want = plan_reference(cached, [added] * n, block, tables, free, 4 * n, tokens)
    want["slots"] = [s if 0 <= s < len(free) * block else -1 for s in want["slots"]]
    got = _plan(cached, [added] * n, block, tables, free, 4 * n, tokens)
    for k, v in want.items():
        assert np.array_equal(got[k], v), k


# ------------------------------------------------------------------ heads of q and k ----
def _randn(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _check_heads(got, want, mag):
    """One rounding to bf16; before it fp32: sum of squares, square root, quotient, two products with inv and gain, cosine, sine,
    two products and a sum: at most dh/8 + 4 + 16 roundings of 2^-24 of each of the two products."""
    tol = 2.0 ** -8 * want.abs() + 40 * 2.0 ** -24 * mag + 1e-30
    err = (got.double().cpu() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@gpu
@pytest.mark.parametrize("norm,theta", [((True, True), 10000.0), ((False, False), 10000.0), ((True, True), 0.0), ((True, False), 5e5), ((False, True), 0.0)])
@pytest.mark.parametrize("T,H,Hk,dh,seq", [(1, 1, 1, 128, 1), (1, 32, 32, 128, 7), (37, 5, 3, 128, 10), (9, 12, 2, 64, 4), (2, 3, 1, 64, 1), (5000, 4, 2, 64, 333)])
def test_heads_without_a_cache(T, H, Hk, dh, seq, norm, theta):
    x = _randn(T, H + 2 * Hk, dh, seed=T + H) * 3
    gains = [(1 + 0.3 * _randn(dh, seed=9 + i).float()).to(torch.bfloat16) if norm[i] else None for i in range(2)]
    at = torch.arange(T) % seq
    parts = [norm_reference(x.double()[:, :H], gains[0], 1e-5), norm_reference(x.double()[:, H:H + Hk], gains[1], 1e-5)]
    want, mag = rope_reference(torch.cat(parts, 1), at, theta)
    dev = x.to(DEV).view(T, -1)
    out = torch.full((T, (H + Hk) * dh + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    g = [None if v is None else v.to(DEV) for v in gains]
    qb.qzo_qk_norm_rope(dev, H, Hk, out, g[0], g[1], 1e-5, theta, seq=seq)
    _check_heads(out[:, :-8].reshape(T, H + Hk, dh), want, mag)
    assert bool((out[:, -8:] == 7.0).all())
    again = torch.empty_like(out)
    qb.qzo_qk_norm_rope(dev, H, Hk, again, g[0], g[1], 1e-5, theta, positions=at.to(torch.int32).to(DEV))
    assert torch.equal(again[:, :-8], out[:, :-8])
    v = dev[:, (H + Hk) * dh:].clone()
    qb.qzo_qk_norm_rope(dev, H, Hk, dev, g[0], g[1], 1e-5, theta, seq=seq)           # in place: v stays
    assert torch.equal(dev[:, :(H + Hk) * dh], out[:, :-8]) and torch.equal(dev[:, (H + Hk) * dh:], v)


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,H,Hk,dh,block,scaled", [(1, 32, 32, 128, 16, True), (33, 6, 2, 64, 32, True), (300, 8, 1, 128, 256, False), (4100, 3, 3, 64, 64, True)])
def test_heads_into_the_cache(T, H, Hk, dh, block, scaled, e4m3):
    """Positions up to 2^30, strided rows, rows without a slot, values beyond e4m3's range."""
    x = _randn(T, H + 2 * Hk, dh, seed=T) * 2
    gains = [(1 + 0.3 * _randn(dh, seed=19 + i).float()).to(torch.bfloat16) for i in range(2)]
    n_blocks = -(-T // block) + 2
    g = torch.Generator().manual_seed(5)
    slots = torch.randperm(n_blocks * block, generator=g)[:T].to(torch.int32)
    at = torch.randint(0, 1 << 30, (T,), generator=g, dtype=torch.int32)
    skip = torch.zeros(T, dtype=torch.bool)
    if T > 3:
        slots[1], slots[2], slots[T - 1] = -1, n_blocks * block, 2 ** 31 - 1
        skip[[1, 2, T - 1]] = True
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    pools = [torch.full((n_blocks, Hk, block, dh), 3.0, device=DEV).to(dtype) for _ in range(2)]
    scales = [torch.linspace(0.003, 0.4, Hk, device=DEV), torch.linspace(1.5, 0.002, Hk, device=DEV)] if e4m3 and scaled else [None, None]
    wide = torch.full((T, (H + 2 * Hk) * dh + 16), 5.0, dtype=torch.bfloat16, device=DEV)
    wide[:, :-16] = x.view(T, -1).to(DEV)
    out = torch.full((T, H * dh), 7.0, dtype=torch.bfloat16, device=DEV)
    qb.qzo_qk_norm_rope(wide[:, :-16], H, Hk, out, gains[0].to(DEV), gains[1].to(DEV), 1e-6, 10000.0, positions=at.to(DEV),
                        cache=qb.make_cache(*pools, *scales), slots=slots.to(DEV))
    q, qm = rope_reference(norm_reference(x.double()[:, :H], gains[0], 1e-6), at, 10000.0)
    k, km = rope_reference(norm_reference(x.double()[:, H:H + Hk], gains[1], 1e-6), at, 10000.0)
    got = out.cpu().view(T, H, dh)
    assert bool((got[skip] == 7.0).all())
    _check_heads(got[~skip], q[~skip], qm[~skip])
    rows = slots[~skip].long()
    for pool, scale, want, mag in ((pools[0], scales[0], k, km), (pools[1], scales[1], x.double()[:, H + Hk:], None)):
        flat = pool.float().cpu().transpose(1, 2).reshape(-1, Hk, dh)
        rest = torch.ones(flat.shape[0], dtype=torch.bool)
        rest[rows] = False
        assert bool((flat[rest] == 3.0).all())
        if not e4m3:
            if mag is None:
                assert torch.equal(flat[rows].double(), want[~skip])
            else:
                _check_heads(flat[rows], want[~skip], mag[~skip])
            continue
        by = 1.0 if scale is None else scale.double().cpu()[:, None]
        want, mag = (want / by)[~skip], ((want.abs() if mag is None else mag) / by)[~skip]
        # half a step: 2^-4 of the value, 2^-10 below the smallest normal one
        tol = 2.0 ** -4 * want.abs().clamp(max=448) + 2.0 ** -10 + 44 * 2.0 ** -24 * mag
        assert bool(((flat[rows].double() - want.clamp(-448, 448)).abs() <= tol).all())


@gpu
@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("T", [1, 2, 37])
def test_heads_in_place(T, cached):
    """Out is the first columns of qkv's own rows, one row and several, without a cache and with one: as apart, bit for bit."""
    H, Hk, dh = 4, 2, 64
    x = _randn(T, (H + 2 * Hk) * dh, seed=T).to(DEV)
    wide = (H if cached else H + Hk) * dh
    got, want = x.clone(), torch.empty(T, wide, dtype=torch.bfloat16, device=DEV)
    pools = [[torch.zeros(4, Hk, 16, dh, dtype=torch.bfloat16, device=DEV) for _ in range(2)] for _ in range(2)]
    for out, src, pool in ((want, x, pools[0]), (got[:, :wide], got, pools[1])):
        more = dict(cache=qb.make_cache(*pool), slots=_i32(range(T))) if cached else {}
        qb.qzo_qk_norm_rope(src, H, Hk, out, positions=_i32(np.arange(T) + 5), **more)
    assert torch.equal(got[:, :wide], want) and torch.equal(got[:, wide:], x[:, wide:]) and not torch.equal(want, x[:, :wide])
    for a, b in zip(*pools):
        assert torch.equal(a, b)


@gpu
def test_heads_keep_to_themselves():
    """NaN and infinities of a head reach that head's outputs only; a head of zeros stays zero under its norm; no tokens, no writes."""
    x = _randn(3, 4 + 2 * 2, 64, seed=3)
    x[1, 2, 5], x[1, 4, 0], x[0, 7, 9], x[2, 0] = math.nan, math.inf, math.nan, 0
    gain = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(3, 6 * 64, dtype=torch.bfloat16, device=DEV)
    qb.qzo_qk_norm_rope(x.to(DEV).view(3, -1), 4, 2, out, gain, gain, 1e-6, 10000.0, seq=5)
    bad = (~torch.isfinite(out.view(3, 6, 64))).any(-1).cpu()
    want = torch.zeros(3, 6, dtype=torch.bool)
    want[1, 2] = want[1, 4] = True
    assert torch.equal(bad, want) and not bool(out.view(3, 6, 64)[2, 0].any())
    qb.qzo_qk_norm_rope(x.to(DEV).view(3, -1)[:0], 4, 2, out[:0], seq=5)
    # e4m3 keeps NaN, infinities end at the largest value
    pools = [torch.zeros(1, 2, 16, 64, device=DEV).to(torch.float8_e4m3fn) for _ in range(2)]
    x[1, 6, 3], x[1, 6, 4] = math.inf, -math.inf
    qb.qzo_qk_norm_rope(x.to(DEV).view(3, -1), 4, 2, out[:, :256], theta=0.0, cache=qb.make_cache(*pools), slots=_i32([0, 1, 2]))
    v = pools[1].float().cpu()
    assert math.isnan(v[0, 1, 0, 9]) and v[0, 0, 1, 3] == 448 and v[0, 0, 1, 4] == -448 and int(torch.isnan(v).sum()) == 1


# ------------------------------------------------------------------ attention over the cache ----
def _attend(lengths, H, Hk, dh, block, news=None, e4m3=False, scaled=True, seed=0, scale=None, pad_rows=0, extra_blocks=2, spread=2.0, tables=None,
            stride=0, spoil=False, run=True):
    """Runs the call on a shuffled cache; returns it all.  spoil: every position that no row sees is NaN or infinite."""
    g = torch.Generator().manual_seed(seed)
    n, starts = len(lengths), [0]
    for i in range(n):
        starts.append(starts[-1] + (1 if news is None else news[i]))
    need = [-(-length // block) for length in lengths]
    most = max(need + [1])
    ids = torch.randperm(sum(need) + extra_blocks, generator=g)
    if tables is None:
        tables, at = torch.full((n, most), -1, dtype=torch.int32), 0
        for i, b in enumerate(need):
            tables[i, :b] = ids[at:at + b].to(torch.int32)
            at += b
    shape = (sum(need) + extra_blocks, Hk, block, dh)
    pools = [torch.randn(shape, generator=g) for _ in range(2)]
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    if spoil:
        seen = torch.zeros(shape[0], block, dtype=torch.bool)
        for i in range(n):
            at = torch.arange(lengths[i])
            seen[tables[i, at // block].long(), at % block] = True
        for p in pools:
            p.transpose(1, 2)[~seen] = math.nan if e4m3 else torch.tensor([math.nan, math.inf, -math.inf, math.nan]).repeat(dh // 4)
    pools = [(p * (3 if e4m3 else 1)).to(dtype) for p in pools]
    scales = [torch.rand(Hk, generator=g) * 0.3 + 0.1 for _ in range(2)] if e4m3 and scaled else [None, None]
    rows = starts[-1] + pad_rows
    q = (torch.randn(rows, H * dh, generator=g) * spread).to(torch.bfloat16)
    scale = dh ** -0.5 if scale is None else scale
    d = dict(lengths=lengths, starts=starts, tables=tables, pools=pools, scales=scales, q=q, scale=scale, dh=dh, H=H)
    d["qd"] = torch.zeros(rows, H * dh + stride, dtype=torch.bfloat16, device=DEV)
    d["qd"][:, :H * dh] = q.to(DEV)
    d["outd"] = torch.full((rows, H * dh + stride), 7.0, dtype=torch.bfloat16, device=DEV)
    d["pd"] = [p.to(DEV) for p in pools]
    d["sd"] = [None if s is None else s.to(DEV) for s in scales]
    d["cache"] = qb.make_cache(*d["pd"], *d["sd"])
    d["args"] = (d["qd"][:, :H * dh], d["cache"], tables.to(DEV), _i32(lengths), d["outd"][:, :H * dh], scale, None if news is None else _i32(starts))
    if run:
        qb.qzo_paged_attention(*d["args"])
    return d


def _check_attend(d):
    k, v = (p.double() if s is None else p.double() * s.double()[:, None, None] for p, s in zip(d["pools"], d["scales"]))
    rows = d["starts"][-1]
    q = d["q"].double().view(-1, d["H"], d["dh"])[:rows]
    at = DEV if rows > 1000 or rows * max(d["lengths"]) * d["H"] > 2e7 else "cpu"
    want, mag, mac = (x.cpu() for x in attention_reference(q.to(at), k.to(at), v.to(at), d["tables"].to(at), d["lengths"], d["starts"], d["scale"]))
    out = d["outd"].cpu()
    got = out[:rows, :d["H"] * d["dh"]].double().view(want.shape)
    tol = attention_tolerance(want, mag, mac, d["dh"])
    err = (got - want).abs()
    assert bool((err <= tol).all()), (float((err / tol).max()), [int(i) for i in (err / tol).nan_to_num(9e9).argmax().unsqueeze(0)])
    assert bool((out[rows:] == 7.0).all()) and bool((out[:, d["H"] * d["dh"]:] == 7.0).all())


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lengths,H,Hk,dh,block", [
    ([1], 1, 1, 128, 16), ([0], 2, 2, 64, 16), ([1, 0, 2, 15, 16, 17], 4, 4, 128, 16), ([31, 32, 33, 63, 64, 65, 0], 4, 2, 64, 32),
    ([127, 128, 129, 255, 256, 257], 6, 2, 128, 64), ([500], 32, 32, 128, 16), ([511, 3], 16, 1, 64, 256), ([700, 33], 40, 8, 128, 128),
    ([300, 1], 34, 2, 64, 32), ([90], 40, 1, 128, 16), ([1025, 2049], 3, 3, 64, 16)])
def test_attention_of_single_tokens(lengths, H, Hk, dh, block, e4m3):
    _check_attend(_attend(lengths, H, Hk, dh, block, e4m3=e4m3, seed=len(lengths) + H))


FEW_COLUMNS = [([40, 25, 60], None, 16, 2, 128), ([40, 25, 60], None, 3, 3, 64), ([20 + i % 40 for i in range(200)], None, 8, 8, 128),
               ([40, 30], [4, 2], 6, 3, 64), ([300], None, 5, 1, 128)]


@gpu
@pytest.mark.parametrize("lengths,news,H,Hk,dh,e4m3", [(*x, e4m3) for x in FEW_COLUMNS for e4m3 in (False, True)] + [
    ([40, 30], None, 24, 2, 64, False), ([60, 40], [60, 12], 4, 2, 64, False)])
def test_weights_of_few_columns_in_two_parts(lengths, news, H, Hk, dh, e4m3):
    """Up to eight columns a sequence and key head (heads that share it, times new tokens), with heads of 64 in bf16 more, too: the weights lose nothing that the output's own
    rounding, half a step of its binade, does not hide.  Before it, for n keys: a weight is two bf16 numbers, the second what the first's
    rounding left, 2^-8 2^-8 of it at most missing, above and below the fraction; its exponential 2^-22; n + 64 sums and products of
    2^-24; scores as everywhere."""
    d = _attend(lengths, H, Hk, dh, 16, news, e4m3=e4m3, seed=H, spread=0.5)
    k, v = (p.double() if s is None else p.double() * s.double()[:, None, None] for p, s in zip(d["pools"], d["scales"]))
    q = d["q"].double().view(-1, H, dh)
    want, mag, mac = attention_reference(q, k, v, d["tables"], lengths, d["starts"], d["scale"])
    before = ((2.0 ** -16 + 2.0 ** -22 + (max(lengths) + 64) * 2.0 ** -24) * (mag + want.abs()) + 2 * (dh + 4) * 2.0 ** -24 * mac[..., None] * mag) * 1.01
    half = torch.exp2(torch.floor(torch.log2((want.abs() + before).clamp(min=1e-30))) - 8)
    err = (d["outd"].double().cpu().view(want.shape) - want).abs()
    assert bool((err <= half + before).all()), float((err / (half + before)).max())


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lengths,news,H,Hk,dh,block", [
    ([5], [5], 2, 2, 128, 16), ([40, 40, 7], [40, 1, 7], 4, 2, 64, 16), ([200, 64, 33], [17, 0, 33], 6, 2, 128, 32), ([20, 0, 130], [3, 0, 129], 16, 1, 64, 16),
    ([3, 5], [6, 2], 4, 4, 64, 16), ([90, 600, 31], [2, 3, 31], 40, 2, 128, 64), ([260], [256], 2, 1, 64, 256)])
def test_attention_of_several_new_tokens(lengths, news, H, Hk, dh, block, e4m3):
    """Causal among the new tokens, sequences that add nothing, more new tokens than the length says (rows that see nothing)."""
    _check_attend(_attend(lengths, H, Hk, dh, block, news, e4m3=e4m3, seed=len(lengths) + H, pad_rows=3, stride=8))


@gpu
@pytest.mark.parametrize("lengths,news,H,Hk,dh,block,e4m3", [
    ([700, 1200, 33, 0, 500], [650, 900, 33, 0, 1], 24, 8, 64, 16, False), ([1500, 70], [1400, 2], 16, 16, 128, 64, False),
    ([1100, 900], [700, 801], 40, 8, 128, 32, True), ([1000, 1024], [900, 1024], 32, 16, 64, 16, False), ([1024, 990], [1024, 950], 32, 16, 64, 32, True)])
def test_attention_of_many_new_tokens(lengths, news, H, Hk, dh, block, e4m3):
    """More than 12288 units of 16 (heads of 64: 32) columns and 128 keys: wide groups; the first has fewer."""
    cols = 16 if dh == 128 else 32
    units = sum(-(-n * (H // Hk) // cols) * Hk * max(1, -(-length // 128)) for length, n in zip(lengths, news))
    assert units >= 12288 or news[0] == 650
    _check_attend(_attend(lengths, H, Hk, dh, block, news, e4m3=e4m3, seed=H, pad_rows=2))
    spoiled, clean = (_attend(lengths, H, Hk, dh, block, news, e4m3=e4m3, seed=H, spoil=s) for s in (True, False))
    assert torch.equal(spoiled["outd"], clean["outd"])


@gpu
@pytest.mark.parametrize("lengths,news,H,Hk,dh,block,e4m3,scale", [
    ([300, 900, 0, 200], [300, 257, 0, 129], 32, 32, 128, 16, False, None), ([1000, 64, 130], [128, 64, 130], 64, 4, 128, 32, True, None),
    ([40, 700], [45, 300], 56, 8, 128, 64, False, -0.05), ([500], [420], 60, 4, 128, 256, True, 0.0), ([4100], [300], 64, 64, 128, 16, False, None),
    ([800, 700], [800, 333], 64, 16, 128, 32, False, None), ([1100, 70], [1024, 70], 64, 16, 64, 16, False, None), ([700, 1500], [600, 500], 64, 2, 64, 64, True, None),
    ([1200], [1100], 60, 4, 64, 128, False, -0.1)])
def test_attention_of_prompts(lengths, news, H, Hk, dh, block, e4m3, scale):
    """At least 96 columns a sequence and more than 128 groups (heads of 64: 511) of 128: keys and values through the LDS.  Whole prompts and
    later parts, more new tokens than the length says, groups of heads that divide 128 and not, groups cut into pieces and not, scales of
    any sign, positions of nobody that hold anything, blocks that are not there."""
    assert sum(news) * H // 128 > (511 if dh == 64 else 128) and sum(news) * (H // Hk) >= 96 * len(news)
    d = _attend(lengths, H, Hk, dh, block, news, e4m3=e4m3, seed=H, pad_rows=2, stride=8, scale=scale)
    _check_attend(d)
    spoiled = _attend(lengths, H, Hk, dh, block, news, e4m3=e4m3, seed=H, pad_rows=2, stride=8, scale=scale, spoil=True)
    assert torch.equal(spoiled["outd"], d["outd"])
    tables = d["tables"].clone()
    tables[0, 0], tables[0, -(-lengths[0] // block) // 2], tables[-1, 0] = -1, 1 << 30, -5
    d = _attend(lengths, H, Hk, dh, block, news, e4m3=e4m3, seed=H, scale=scale, tables=tables, run=False)
    qb.qzo_paged_attention(*d["args"])
    _check_attend(d)


@gpu
@pytest.mark.parametrize("lengths,news,H,Hk,dh", [([700, 333], [600, 333], 32, 8, 128), ([2100], [260], 64, 4, 128), ([1100], [1030], 64, 64, 64)])
def test_captured_prompts_replay(lengths, news, H, Hk, dh):
    """Replays over other queries and other lengths, eager work in between, against eager calls."""
    d = _attend(lengths, H, Hk, dh, 16, news, seed=5, run=False)
    q, cache, tables, at, out, scale, starts = d["args"]
    scratch = torch.zeros(qb.qzo_paged_attention_scratch_bytes(q.shape[0], len(lengths), H, dh), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        qb.qzo_paged_attention(q, cache, tables, at, out, scale, starts, scratch=scratch)
    want = torch.empty_like(out)
    for i in range(4):
        d["qd"].copy_(_randn(*d["qd"].shape, seed=i).to(DEV))
        at.copy_(_i32([n - 37 * i for n in lengths]))
        out.fill_(7.0)
        graph.replay()
        qb.qzo_paged_attention(q, cache, tables, at, want, scale, starts)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and not bool(scratch[:2048].any())


@gpu
def test_attention_of_many_prompts():
    """More sequences than a wavefront has lanes."""
    rng = np.random.default_rng(3)
    news = [int(x) for x in rng.integers(8, 14, 80)]
    lengths = [n + int(x) for n, x in zip(news, rng.integers(0, 300, 80))]
    _check_attend(_attend(lengths, 32, 2, 128, 16, news, seed=8))


@gpu
@pytest.mark.parametrize("n,longest,H,Hk,dh,block,seed", [(300, 40, 4, 4, 64, 16, 1), (70, 900, 8, 8, 128, 32, 2), (9, 9000, 8, 2, 128, 16, 3), (1, 70000, 2, 1, 64, 128, 4),
                                                         (2000, 3, 2, 1, 64, 16, 5)])
def test_attention_of_ragged_batches(n, longest, H, Hk, dh, block, seed):
    """Sequences that are cut into pieces beside ones that are not."""
    rng = np.random.default_rng(seed)
    lengths = [int(x) for x in (longest ** rng.random(n)).round()]
    lengths[0] = longest
    _check_attend(_attend(lengths, H, Hk, dh, block, seed=seed, spread=3.0))


@gpu
@pytest.mark.parametrize("n,longest,new,H,Hk,dh,block,e4m3", [
    (300, 30, 1, 5, 5, 64, 16, False), (130, 600, 1, 6, 6, 128, 32, False), (90, 700, 1, 14, 7, 64, 16, True), (600, 3, 1, 2, 1, 128, 16, False),
    (140, 512, 4, 12, 4, 128, 16, False), (40, 550, 30, 30, 15, 64, 16, False), (520, 1, 1, 1, 1, 64, 16, True), (90, 513, 1, 40, 10, 128, 128, True)])
def test_attention_of_many_short_sequences(n, longest, new, H, Hk, dh, block, e4m3):
    """More groups than workgroups, sequences of up to 512 positions (four key heads a workgroup, their number odd) beside longer ones,
    one and several new tokens, empty sequences."""
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in (longest ** rng.random(n)).round()]
    lengths[0], lengths[n // 2], lengths[-1] = longest, 0, min(longest, 512)
    news = None if new == 1 else [int(x) for x in rng.integers(0, new + 1, n)]
    _check_attend(_attend(lengths, H, Hk, dh, block, news, e4m3=e4m3, seed=n, pad_rows=2))


@gpu
def test_attention_of_more_and_fewer_rows_than_sequences():
    """A row per sequence, with rows behind the last sequence (left as they are), and with sequences that have no row."""
    _check_attend(_attend([40, 0, 300], 4, 2, 64, 16, seed=1, pad_rows=4, stride=16))
    d = _attend([40, 70, 300], 4, 2, 64, 16, seed=1, run=False)
    qb.qzo_paged_attention(d["args"][0][:2], d["cache"], *d["args"][2:4], d["args"][4][:2], d["scale"])
    assert bool((d["outd"][2] == 7.0).all())
    whole = _attend([40, 70, 300], 4, 2, 64, 16, seed=1)
    assert torch.equal(d["outd"][:2], whole["outd"][:2])
    _check_attend(_attend([40, 70], 4, 2, 64, 16, e4m3=True, scaled=False, seed=2))
    for scale in (-0.1, 0.0):
        _check_attend(_attend([40, 700], 8, 2, 128, 16, scale=scale, seed=2))


@gpu
def test_attention_with_room_for_very_long_sequences():
    """Tables whose rows reach 2^29 positions: the units of what might be no longer fit 32 bits."""
    d = _attend([40, 700], 8, 4, 64, 16, seed=5, run=False)
    wide = torch.full((2, 1 << 25), -1, dtype=torch.int32, device=DEV)
    wide[:, :d["tables"].shape[1]] = d["args"][2]
    qb.qzo_paged_attention(*d["args"][:2], wide, *d["args"][3:])
    _check_attend(d)


@gpu
def test_a_row_of_nan_stays_alone():
    for news in (None, [1, 3]):
        clean = _attend([100, 70], 4, 2, 128, 16, news, seed=7)
        d = _attend([100, 70], 4, 2, 128, 16, news, seed=7, run=False)
        d["qd"][1, 130] = math.nan                           # head 1 of row 1
        d["qd"][1, 300] = math.inf                           # head 2
        qb.qzo_paged_attention(*d["args"])
        bad = torch.zeros_like(d["outd"], dtype=torch.bool)
        bad[1, 128:384] = True
        assert not torch.isfinite(d["outd"][bad]).any() and torch.equal(d["outd"][~bad], clean["outd"][~bad])


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lengths,news", [([1, 17, 100, 0, 333], None), ([9, 100, 333], [9, 3, 40])])
def test_unseen_positions_hold_anything(lengths, news, e4m3):
    """The rest of a block, blocks of nobody: NaN and infinities.  The same bits as with zeros there."""
    d = _attend(lengths, 4, 2, 64, 32, news, e4m3=e4m3, seed=3, spoil=True)
    clean = _attend(lengths, 4, 2, 64, 32, news, e4m3=e4m3, seed=3)
    assert torch.equal(d["outd"], clean["outd"])
    _check_attend(clean)


@gpu
@pytest.mark.parametrize("length,new,at,H,Hk,dh", [(70, 20, 61, 4, 2, 64), (70, 20, 61, 2, 1, 128), (40, 3, 38, 6, 1, 128), (1300, 1100, 777, 32, 16, 64),
                                                    (700, 300, 501, 64, 32, 128), (1300, 1100, 777, 64, 32, 64)])
def test_later_tokens_hold_anything(length, new, at, H, Hk, dh):
    """A new token's key and value are NaN or infinite: the rows before it do not see it, its own and the later ones do."""
    clean = _attend([length], H, Hk, dh, 16, [new], seed=4)
    first = at - (length - new)
    for which, what in ((1, math.nan), (1, math.inf), (0, math.nan)):
        d = _attend([length], H, Hk, dh, 16, [new], seed=4, run=False)
        d["pd"][which][int(d["tables"][0, at // 16]), :, at % 16] = what
        qb.qzo_paged_attention(*d["args"])
        got = d["outd"].cpu()
        assert torch.equal(got[:first], clean["outd"].cpu()[:first])
        assert not torch.isfinite(got[first:]).any()


@gpu
@pytest.mark.parametrize("lengths,news,H,Hk,dh,e4m3", [
    ([700, 33, 1], None, 8, 2, 128, False), ([700, 33, 1], None, 8, 2, 64, True), ([50 + i for i in range(80)], None, 16, 8, 128, False),
    ([400, 90], [100, 60], 8, 2, 64, False), ([400, 90], [100, 60], 8, 2, 128, True), ([9000] * 6, [8] * 6, 64, 8, 128, False),
    ([700, 333], [600, 333], 32, 8, 128, False), ([1100], [1030], 64, 32, 64, True), ([1100], [1030], 64, 32, 64, False)])
def test_scores_of_minus_infinity_hide_a_key(lengths, news, H, Hk, dh, e4m3):
    """A score that leaves fp32 downwards counts as unseen: for the heads that have it, what such a key's value holds reaches nothing; the heads
    beside them see it.  Narrow, wide and four key heads' groups, 32 columns, prompts."""
    hidden, f = [0, 3, 31, 32, 40, 127, 128, 300, 9000 - 1], 5
    got = []
    for what in (1.0, math.nan, math.nan if e4m3 else math.inf):
        d = _attend(lengths, H, Hk, dh, 16, news, e4m3=e4m3, seed=H + dh, run=False)
        q = d["qd"].view(-1, H, dh)
        q[..., f] = 0
        q[:, 1::2, f] = 2.0 ** 127                       # times 448: beyond fp32
        d["q"] = d["qd"].cpu()
        d["pd"][0].view(torch.uint8 if e4m3 else torch.int16)[..., f] = 0
        for i, length in enumerate(lengths):
            for at in hidden:
                if at < length:
                    b = int(d["tables"][i, at // 16])
                    d["pd"][0][b, :, at % 16, f] = -448.0
                    d["pd"][1][b, :, at % 16] = what
        qb.qzo_paged_attention(*d["args"])
        got.append(d["outd"].view(-1, H, dh).clone())
        if what != 1.0 or sum(lengths) > 2000:
            continue
        # against 64 bits: the hidden keys masked, without the feature that hides them
        k, v = (p.double().cpu() if s is None else p.double().cpu() * s.double()[:, None, None] for p, s in zip(d["pd"], d["scales"]))
        at = torch.arange(max(lengths))
        for i, length in enumerate(lengths):
            ids = d["tables"][i, at[:length] // 16].long()
            for r in range(d["starts"][i], d["starts"][i + 1]):
                sees = length - (d["starts"][i + 1] - 1 - r)
                seen = torch.tensor([p for p in range(sees) if p not in hidden], dtype=torch.long)
                if seen.numel() == 0:
                    assert not bool(got[0][r, 1::2].any())
                    continue
                kk, vv = (p[ids[seen], :, seen % 16].repeat_interleave(H // Hk, 1)[:, 1::2] for p in (k, v))
                kk[..., f] = 0
                qq = d["q"].double().view(-1, H, dh)[r, 1::2]
                p = torch.softmax(d["scale"] * (qq * kk).sum(-1), 0)
                want, mag = (p[..., None] * vv).sum(0), (p[..., None] * vv.abs()).sum(0)
                mac = (d["scale"] * (qq.abs() * kk.abs()).sum(-1)).amax(0)
                assert bool(((got[0][r, 1::2].double().cpu() - want).abs() <= attention_tolerance(want, mag, mac, dh)).all()), (i, r)
    assert bool(torch.isfinite(got[0]).all())
    for spoiled in got[1:]:
        assert torch.equal(spoiled[:, 1::2], got[0][:, 1::2])
        assert not bool(torch.isfinite(spoiled[:, 0::2]).any())


@gpu
def test_blocks_outside_the_pool_are_absent():
    tables = torch.tensor([[3, -1, 1, 99], [2 ** 31 - 1, -2 ** 31, 4, 5], [-1, -1, -1, -1]], dtype=torch.int32)
    d = _attend([60, 64, 50], 4, 2, 64, 16, seed=6, tables=tables, extra_blocks=0)
    _check_attend(d)
    assert not bool(d["outd"][2].any())
    # lengths beyond the table's reach
    d = _attend([60], 4, 2, 64, 16, seed=6, run=False)
    d["lengths"] = [2 ** 31 - 1]
    qb.qzo_paged_attention(d["args"][0], d["args"][1], d["args"][2], _i32(d["lengths"]), *d["args"][4:])
    _check_attend(d)
    # a negative length sees nothing
    qb.qzo_paged_attention(d["args"][0], d["args"][1], d["args"][2], _i32([-3]), *d["args"][4:])
    assert not bool(d["outd"].any())


@gpu
@pytest.mark.parametrize("dh", [64, 128])
def test_large_and_sharp_scores(dh):
    """Scores of some +-1500 of either sign of the scale: one key takes all."""
    for sign in (1.0, -1.0):
        _check_attend(_attend([1000, 333], 4, 2, dh, 16, seed=8, scale=sign * 20.0, spread=3.0))
    d = _attend([50], 2, 2, dh, 16, seed=9, scale=0.0)            # all keys alike: the mean of the values
    _check_attend(d)


@gpu
def test_cache_beyond_32_bits():
    """Pools of 4.3 GB each, the sequence's blocks at their end."""
    Hk, dh, block = 8, 128, 64
    n_blocks = (1 << 32) // (Hk * dh * block * 2) + 40
    pools = [torch.empty(n_blocks, Hk, block, dh, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ids = torch.tensor([[n_blocks - 1, 0, n_blocks - 7, n_blocks // 2 + 1]], dtype=torch.int32)
    x = _randn(250, (Hk + 2 * Hk) * dh, seed=2).to(DEV)
    slots = (ids[0].long().repeat_interleave(block)[:250] * block + torch.arange(250) % block).to(torch.int32)
    q = torch.empty(250, Hk * dh, dtype=torch.bfloat16, device=DEV)
    cache = qb.make_cache(*pools)
    qb.qzo_qk_norm_rope(x, Hk, Hk, q, theta=0.0, cache=cache, slots=slots.to(DEV))
    heads = x.view(250, 3 * Hk, dh)
    assert torch.equal(q, x[:, :Hk * dh])
    for pool, part in zip(pools, (heads[:, Hk:2 * Hk], heads[:, 2 * Hk:])):
        assert torch.equal(pool[slots.long().to(DEV) // block, :, slots.long().to(DEV) % block], part)
    out = torch.empty(1, Hk * dh, dtype=torch.bfloat16, device=DEV)
    qb.qzo_paged_attention(q[249:], cache, ids.to(DEV), _i32([250]), out, dh ** -0.5)
    small = [torch.zeros(4, Hk, block, dh, dtype=torch.bfloat16) for _ in range(2)]
    for p, part in zip(small, (heads[:, Hk:2 * Hk], heads[:, 2 * Hk:])):
        p.transpose(1, 2).reshape(-1, Hk, dh)[:250] = part.cpu()
        p[:] = torch.nn.functional.pad(part.cpu(), (0, 0, 0, 0, 0, 6)).view(4, block, Hk, dh).transpose(1, 2)
    want, mag, mac = attention_reference(q[249:].double().cpu().view(1, Hk, dh), small[0].double(), small[1].double(),
                                         torch.arange(4, dtype=torch.int32)[None], [250], [0, 1], dh ** -0.5)
    assert bool(((out.double().cpu().view(want.shape) - want).abs() <= attention_tolerance(want, mag, mac, dh)).all())


# ------------------------------------------------------------------ as they are used ----
def _layer_inputs(tokens, H, Hk, dh, seed):
    return (_randn(tokens, (H + 2 * Hk) * dh, seed=seed)).to(DEV)


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_sequences_are_continued(e4m3):
    """Prompts of different lengths come in, are continued token by token while one ends and another comes in: every step's
    output is the attention over the sequence's own keys and values, kept here in plain lists."""
    H, Hk, dh, block, n, most, blocks, pad = 6, 2, 64, 16, 4, 8, 20, 64
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    pools = [torch.zeros(blocks, Hk, block, dh, device=DEV).to(dtype) for _ in range(2)]
    cache = qb.make_cache(*pools)
    gains = [(1 + 0.2 * _randn(dh, seed=i).float()).to(torch.bfloat16).to(DEV) for i in range(2)]
    tables, free, state = _i32(np.full((n, most), -1)), _i32(np.arange(blocks)), _i32([blocks, 0, 0, 0])
    lengths, starts, slots, positions = _i32([0] * n), _i32([0] * (n + 1)), _i32([0] * pad), _i32([0] * pad)
    kept = [[[], []] for _ in range(n)]
    steps = [[30, 1, 17, 0], [1, 1, 1, 16], [1, 1, -1, 1], [1, 1, 9, 1], [0, 1, 1, -1], [1, 1, 1, 33]] + [[1, 1, 1, 1]] * 3
    for number, added in enumerate(steps):
        x = _layer_inputs(pad, H, Hk, dh, 50 + number)
        q = torch.full((pad, H * dh), 7.0, dtype=torch.bfloat16, device=DEV)
        out = torch.full((pad, H * dh), 7.0, dtype=torch.bfloat16, device=DEV)
        qb.qzo_cache_plan(lengths, _i32(added), block, tables, free, state, lengths, starts, slots, positions, state)
        qb.qzo_qk_norm_rope(x, H, Hk, q, *gains, positions=positions, cache=cache, slots=slots)
        qb.qzo_paged_attention(q, cache, tables, lengths, out, dh ** -0.5, starts=starts)
        assert state.tolist()[2] == 0
        at = 0
        heads = x.double().cpu().view(pad, H + 2 * Hk, dh)
        for i, a in enumerate(added):
            if a < 0:
                kept[i] = [[], []]
            for _ in range(max(0, a)):
                p = torch.tensor([len(kept[i][0])])
                qq, kk = (rope_reference(norm_reference(heads[at:at + 1, s], g.cpu(), 1e-6), p, 10000.0)[0] for s, g in
                          ((slice(0, H), gains[0]), (slice(H, H + Hk), gains[1])))
                kept[i][0].append(kk[0])
                kept[i][1].append(heads[at, H + Hk:])
                k, v = (torch.stack(c).repeat_interleave(H // Hk, 1) for c in kept[i])
                w = torch.softmax((qq * k).sum(-1) * dh ** -0.5, 0)
                want, mag = (w[..., None] * v).sum(0), (w[..., None] * v.abs()).sum(0)
                # q and k are rounded (2^-8 each) on their way into a score, in e4m3 k (and v) by 2^-4 + 2^-10
                mac = (qq.abs() * k.abs()).sum(-1).amax(0) * dh ** -0.5
                kstep = 2.0 ** -4 + 2.0 ** -8 if e4m3 else 2.0 ** -8
                tiny = 2.0 ** -10 if e4m3 else 0.0
                ds = (2.0 ** -8 + kstep) * mac + tiny * qq.abs().sum(-1)[0] * dh ** -0.5 + 1e-4
                tol = 2.0 ** -8 * want.abs() + ((torch.exp(2 * ds) - 1)[:, None] + 2.0 ** -8 + (kstep if e4m3 else 0)) * mag + tiny
                got = out[at].double().cpu().view(H, dh)
                assert bool(((got - want).abs() <= tol).all()), (number, i)
                at += 1
        assert bool((out[at:] == 7.0).all()) and bool((q[at:] == 7.0).all())
    held = (lengths + block - 1) // block
    in_use = [int(t) for i in range(n) for t in tables[i, :int(held[i])]]
    rest = free[:int(state[0])].tolist()
    assert sorted(in_use + rest) == list(range(blocks))              # every block is somebody's, once


@gpu
def test_captured_steps_replay():
    """A step captured into a graph goes on from the state that its replays leave, as the same calls do one by one."""
    H, Hk, dh, block, n, most, blocks = 4, 2, 128, 16, 3, 16, 40

    def fresh():
        d = dict(pools=[torch.zeros(blocks, Hk, block, dh, dtype=torch.bfloat16, device=DEV) for _ in range(2)], tables=_i32(np.full((n, most), -1)),
                 free=_i32(np.arange(blocks)), state=_i32([blocks, 0, 0, 0]), lengths=_i32([0] * n), starts=_i32([0] * (n + 1)), slots=_i32([0] * n),
                 positions=_i32([0] * n), added=_i32([1] * n), x=torch.zeros(n, (H + 2 * Hk) * dh, dtype=torch.bfloat16, device=DEV),
                 q=torch.zeros(n, H * dh, dtype=torch.bfloat16, device=DEV), out=torch.zeros(n, H * dh, dtype=torch.bfloat16, device=DEV))
        d["cache"] = qb.make_cache(*d["pools"])
        d["scratch"] = torch.zeros(max(256, qb.qzo_paged_attention_scratch_bytes(n, n, H, dh)), dtype=torch.uint8, device=DEV)
        return d

    def step(d):
        qb.qzo_cache_plan(d["lengths"], d["added"], block, d["tables"], d["free"], d["state"], d["lengths"], d["starts"], d["slots"], d["positions"], d["state"])
        qb.qzo_qk_norm_rope(d["x"], H, Hk, d["q"], positions=d["positions"], cache=d["cache"], slots=d["slots"])
        qb.qzo_paged_attention(d["q"], d["cache"], d["tables"], d["lengths"], d["out"], dh ** -0.5, scratch=d["scratch"])

    one, two = fresh(), fresh()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(two)
    for t in range(50):
        x = _randn(n, (H + 2 * Hk) * dh, seed=t).to(DEV)
        for d in (one, two):
            d["x"].copy_(x)
        step(one)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(one["out"], two["out"]) and torch.equal(one["state"], two["state"]), t
        assert one["lengths"].tolist() == [t + 1] * n
    assert torch.equal(one["pools"][0], two["pools"][0]) and torch.equal(one["tables"], two["tables"])


@gpu
def test_calls_on_two_streams_at_once():
    """Two streams with calls of their own, scratch by stream: both as one by one; and a capture without scratch is refused."""
    a = _attend([3000, 700, 50], 8, 2, 128, 32, seed=1)
    b = _attend([2000, 64, 1900, 3], 8, 4, 64, 16, seed=2)
    torch.cuda.synchronize()
    want = [a["outd"].clone(), b["outd"].clone()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, d in zip(streams, (a, b)):
            qb.qzo_paged_attention(*d["args"], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(a["outd"], want[0]) and torch.equal(b["outd"], want[1])
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        a["outd"].zero_()
        with pytest.raises(AssertionError):
            qb.qzo_paged_attention(*a["args"])


@gpu
def test_calls_of_two_threads():
    """Two threads, each with a stream of its own, whose calls need different amounts of LDS: both run, with the results that they have alone."""
    calls = []
    for n, seed in ((8192, 1), (6000, 2)):
        d = _attend([1 + i % 3 for i in range(n)], 1, 1, 64, 16, seed=seed)
        calls.append((d, d["outd"].clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    failed = []

    def work(d, stream):
        try:
            scratch = torch.zeros(qb.qzo_paged_attention_scratch_bytes(d["qd"].shape[0], len(d["lengths"]), 1, 64), dtype=torch.uint8, device=DEV)
            torch.cuda.synchronize()
            for _ in range(3000):
                qb.qzo_paged_attention(*d["args"], scratch=scratch, stream=stream)
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(d, stream)) for d, _, stream in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed and all(torch.equal(d["outd"], want) for d, want, _ in calls)


@gpu
def test_a_capture_on_a_passed_stream_needs_scratch_of_its_own():
    """The stream that is captured is passed while another one is the current one, and the other way round."""
    d = _attend([100, 40], 4, 2, 64, 16, seed=1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        captured = torch.cuda.current_stream()
        d["outd"].zero_()
        with torch.cuda.stream(side), pytest.raises(AssertionError):
            qb.qzo_paged_attention(*d["args"], stream=captured)
        with pytest.raises(AssertionError):
            qb.qzo_paged_attention(*d["args"], stream=side)
    torch.cuda.synchronize()


@gpu
def test_scratch_elsewhere_is_refused():
    """Host memory, and memory with gaps."""
    d = _attend([100], 4, 2, 64, 16, seed=1)
    need = qb.qzo_paged_attention_scratch_bytes(1, 1, 4, 64)
    before = d["outd"].clone()
    for bad in (torch.zeros(need, dtype=torch.uint8), torch.zeros(need, dtype=torch.uint8).pin_memory(), torch.zeros(2 * need, dtype=torch.uint8, device=DEV)[::2]):
        with pytest.raises(AssertionError):
            qb.qzo_paged_attention(*d["args"], scratch=bad)
    torch.cuda.synchronize()
    assert torch.equal(before, d["outd"])


@gpu
def test_scratch_that_is_too_small_is_refused():
    d = _attend([100], 4, 2, 64, 16, seed=1)
    need = qb.qzo_paged_attention_scratch_bytes(1, 1, 4, 64)
    before = d["outd"].clone()
    for small in (torch.zeros(need - 1, dtype=torch.uint8, device=DEV), None):
        with pytest.raises(qb.QzoError):
            qb.qzo_paged_attention(*d["args"], scratch=small)
    torch.cuda.synchronize()
    assert torch.equal(before, d["outd"])
