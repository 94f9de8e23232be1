"""Sequences that fork: the next beams, tables that share blocks, a pool made compact, copied blocks, attention behind what a group has in
common, against plain implementations in 64 bits (whole numbers: equal).

Tolerances are what the roundings add up to.  eps/2 of bf16 is 2^-8, of e4m3 2^-4, of fp32 2^-24."""
import ctypes as C
import math
import random
import types

import numpy as np
import pytest
import torch

from paper_2505_13430_amd import binding as qb
from paper_2505_13430_amd.model import Answers, Beams
from test_answers import _apart, _far, _logits, _model
from test_paged_cache import BAD_CACHES, _cache, _i32, _p, attention_reference, attention_tolerance

DEV = "cuda:0"
gpu = pytest.mark.gpu


# ------------------------------------------------------------------ plain implementations ----
def fork_reference(parents, lengths, tables, free, n_free, block, group_starts=()):
    """tables, free numpy; returns a status or what the call leaves."""
    n, most = tables.shape
    if n_free < 0 or n_free > len(free) or max(parents) >= n or min(lengths) < 0:
        return qb.QZO_ERR_ARG
    if max(lengths) > most * block:
        return qb.QZO_ERR_SHAPE
    rows = [list(tables[i, :-(-lengths[i] // block)]) for i in range(n)]
    stack, seen = list(free[:n_free]), set()
    for p in parents:
        if p >= 0:
            seen |= set(rows[p])
    for i in range(n):
        if i not in parents:
            for b in rows[i]:
                if b not in seen and 0 <= b < len(free):
                    seen.add(b)
                    stack.append(b)
    if len(stack) > len(free):
        return qb.QZO_ERR_ARG
    top, used, copies, after, length = len(stack), set(), [], tables.copy(), []
    for i, p in enumerate(parents):
        if p < 0:
            length.append(0)
            continue
        row = list(rows[p])
        if lengths[p] % block and p in used:
            if not stack:
                return qb.QZO_ERR_WORKSPACE
            copies.append([row[-1], stack[-1], lengths[p] % block, 0])
            row[-1] = stack.pop()
        used.add(p)
        after[i, :len(row)] = row
        length.append(lengths[p])
    out_free = free.copy()
    out_free[n_free:len(stack)] = stack[n_free:]
    return dict(lengths=length, tables=after, free=out_free, state=[len(stack), 0, 0, len(copies)], copies=copies,
                shared=shared_reference(length, after, block, group_starts))


def shared_reference(lengths, tables, block, group_starts):
    out = []
    for a, b in zip(group_starts[:-1], group_starts[1:]):
        live, k = [i for i in range(a, b) if lengths[i] > 0], 0
        while live and all(k < lengths[i] // block for i in live) and len({int(tables[i, k]) for i in live}) == 1:
            k += 1
        out.append(k * block)
    return out


def select_reference(logits, width, scores, counts, ended, history, end, alpha):
    """logits fp64 [rows, vocab]; everything else lists.  Returns rows' outputs and the smallest distance of two keys that decides anything."""
    rows, V = logits.shape
    out = dict(scores=[], counts=[], ended=[], parents=[], chosen=[], added=[], history=history.copy())
    gap = math.inf
    for g in range(rows // width):
        found = []
        for b in range(width):
            r = g * width + b
            s, n = float(scores[r]), max(0, counts[r])
            if not s > -math.inf:
                continue
            if ended[r]:
                found.append((s / max(1, n) ** alpha, -(b * V + max(end, 0)), s))
                continue
            x = np.where(np.isfinite(logits[r]), logits[r], -np.inf)
            if not np.isfinite(x).any():
                continue
            total = x - (np.log(np.exp(x - x.max()).sum()) + x.max()) + s
            for v in np.argsort(-x, kind="stable")[:width + 1]:
                if np.isfinite(x[v]):
                    found.append((total[v] / (n + 1) ** alpha, -(b * V + int(v)), total[v]))
        found.sort(reverse=True)
        for x, y in zip(found[:width], found[1:width + 1]):
            same_beam = -x[1] // V == -y[1] // V
            gap = min(gap, math.inf if same_beam else x[0] - y[0] or math.inf)
        for i in range(width):
            row = g * width + i
            if i >= len(found):
                for name, v in (("scores", -math.inf), ("counts", 0), ("ended", 1), ("parents", -1), ("chosen", -1), ("added", 0)):
                    out[name].append(v)
                continue
            _, place, total = found[i]
            p, v = g * width + -place // V, -place % V
            n, was = max(0, counts[p]), bool(ended[p])
            done = was or v == end
            for name, x in (("scores", total), ("counts", n + (not was)), ("ended", int(done)), ("parents", p), ("chosen", v), ("added", int(not done))):
                out[name].append(x)
            out["history"][row, :n] = history[p, :n]
            if not was and n < history.shape[1]:
                out["history"][row, n] = v
    tokens = [v for v, on in zip(out["chosen"], out["added"]) if on]
    out["tokens"] = tokens + [0] * (rows - len(tokens))
    return out, gap


# ------------------------------------------------------------------ refusals, on the host ----
@pytest.mark.parametrize("over,status", [
    (dict(parents=None), qb.QZO_ERR_ARG), (dict(copies=None), qb.QZO_ERR_ARG), (dict(groups=1), qb.QZO_ERR_ARG), (dict(starts=16), qb.QZO_ERR_ARG),
    (dict(groups=1, starts=16, shared=24), qb.QZO_ERR_ALIGN), (dict(tables=24), qb.QZO_ERR_ALIGN), (dict(n_seq=0), qb.QZO_ERR_SHAPE),
    (dict(n_seq=8193), qb.QZO_ERR_SHAPE), (dict(block=17), qb.QZO_ERR_SHAPE), (dict(block=512), qb.QZO_ERR_SHAPE), (dict(n_blocks=0), qb.QZO_ERR_SHAPE),
    (dict(n_blocks=1 << 27), qb.QZO_ERR_SHAPE), (dict(max_blocks=0), qb.QZO_ERR_SHAPE), (dict(n_seq=4096, max_blocks=1 << 19), qb.QZO_ERR_SHAPE),
    (dict(max_blocks=1 << 27), qb.QZO_ERR_SHAPE), (dict(groups=3, starts=16, shared=16), qb.QZO_ERR_SHAPE), (dict(scratch=None), qb.QZO_ERR_ARG),
    (dict(scratch=128), qb.QZO_ERR_ALIGN), (dict(bytes=64), qb.QZO_ERR_WORKSPACE)])
def test_fork_refuses(over, status):
    v = dict(parents=16, n_seq=2, block=16, n_blocks=8, max_blocks=4, lengths=16, tables=16, free=16, state=16, groups=0, starts=None, shared=None, copies=16,
             scratch=256, bytes=1 << 20)
    v.update(over)
    assert qb.lib().qzo_cache_fork(*v.values(), None) == status and qb.lib().qzo_last_error()


@pytest.mark.parametrize("over,status", [
    (dict(lengths=None), qb.QZO_ERR_ARG), (dict(new=None), qb.QZO_ERR_ARG), (dict(copies=8), qb.QZO_ERR_ALIGN), (dict(n_seq=0), qb.QZO_ERR_SHAPE), (dict(block=8), qb.QZO_ERR_SHAPE),
    (dict(n_blocks=0), qb.QZO_ERR_SHAPE), (dict(scratch=None), qb.QZO_ERR_ARG), (dict(scratch=264), qb.QZO_ERR_ALIGN), (dict(bytes=0), qb.QZO_ERR_WORKSPACE)])
def test_compact_refuses(over, status):
    v = dict(n_seq=2, block=16, n_blocks=8, max_blocks=4, lengths=16, tables=16, new=16, free=16, state=16, copies=16, scratch=256, bytes=1 << 20)
    v.update(over)
    assert qb.lib().qzo_cache_compact(*v.values(), None) == status and qb.lib().qzo_last_error()


@pytest.mark.parametrize("over,status", BAD_CACHES + [
    (dict(_layers=0), qb.QZO_ERR_SHAPE), (dict(_layers=65536), qb.QZO_ERR_SHAPE), (dict(_copies=None), qb.QZO_ERR_ARG), (dict(_copies=24), qb.QZO_ERR_ALIGN),
    (dict(_n=1 << 31), qb.QZO_ERR_SHAPE), (dict(_count=18), qb.QZO_ERR_ALIGN), (dict(kv_heads=65535, _layers=65535), qb.QZO_ERR_SHAPE)])
def test_copy_refuses(over, status):
    v = dict(_layers=2, _copies=16, _n=3, _count=None)
    v.update({k: x for k, x in over.items() if k in v})
    c = _cache(**{k: x for k, x in over.items() if k not in v})
    assert qb.lib().qzo_cache_copy(C.addressof(c), *v.values(), None) == status and qb.lib().qzo_last_error()
    assert qb.lib().qzo_cache_copy(None, 1, 16, 1, None, None) == qb.QZO_ERR_ARG


@pytest.mark.parametrize("over,status", [
    (dict(logits=None), qb.QZO_ERR_ARG), (dict(added=None), qb.QZO_ERR_ARG), (dict(history=None), qb.QZO_ERR_ARG), (dict(columns=0), qb.QZO_ERR_ARG),
    (dict(logits=17), qb.QZO_ERR_ALIGN), (dict(scores=24), qb.QZO_ERR_ALIGN), (dict(groups=0), qb.QZO_ERR_SHAPE), (dict(width=0), qb.QZO_ERR_SHAPE),
    (dict(width=65), qb.QZO_ERR_SHAPE), (dict(groups=2049), qb.QZO_ERR_SHAPE), (dict(vocab=0), qb.QZO_ERR_SHAPE), (dict(vocab=(1 << 22) + 1, ld=1 << 23), qb.QZO_ERR_SHAPE),
    (dict(ld=99), qb.QZO_ERR_SHAPE), (dict(end=100), qb.QZO_ERR_ARG), (dict(end=-2), qb.QZO_ERR_ARG), (dict(alpha=-0.5), qb.QZO_ERR_ARG),
    (dict(alpha=math.nan), qb.QZO_ERR_ARG), (dict(scratch=None), qb.QZO_ERR_ARG), (dict(bytes=16), qb.QZO_ERR_WORKSPACE)])
def test_select_refuses(over, status):
    v = dict(logits=16, ld=100, groups=2, width=4, vocab=100, end=-1, alpha=0.0, scores=16, counts=16, ended=16, history=16, columns=5, parents=16, chosen=16, tokens=16,
             added=16, scratch=256, bytes=1 << 20)
    v.update(over)
    assert qb.lib().qzo_beam_select(*v.values(), None) == status and qb.lib().qzo_last_error()


@pytest.mark.parametrize("over,status", [
    (dict(q=None), qb.QZO_ERR_ARG), (dict(group_starts=None), qb.QZO_ERR_ARG), (dict(shared=None), qb.QZO_ERR_ARG), (dict(shared=20), qb.QZO_ERR_ALIGN),
    (dict(groups=0), qb.QZO_ERR_SHAPE), (dict(groups=2049), qb.QZO_ERR_SHAPE), (dict(q_heads=3), qb.QZO_ERR_SHAPE), (dict(n_seq=0), qb.QZO_ERR_SHAPE),
    (dict(ld_q=264), qb.QZO_ERR_ARG), (dict(ld_q=252), qb.QZO_ERR_SHAPE), (dict(scale=math.inf), qb.QZO_ERR_ARG), (dict(scratch=None), qb.QZO_ERR_ARG),
    (dict(bytes=4096), qb.QZO_ERR_WORKSPACE)])
def test_shared_attention_refuses(over, status):
    c = _cache()
    v = dict(q=16, ld_q=256, n_rows=2, n_seq=2, q_heads=4, cache=C.addressof(c), tables=16, max_blocks=4, lengths=16, starts=None, groups=1, group_starts=16, shared=16,
             scale=0.1, out=16, ld_out=256, scratch=256, bytes=1 << 30)
    v.update(over)
    if over == dict(ld_q=264):          # a longer row is fine: what is refused is the next argument
        v["scale"] = math.nan
    assert qb.lib().qzo_paged_attention_shared(*v.values(), None) == status and qb.lib().qzo_last_error()


@pytest.mark.parametrize("over", BAD_CACHES)
def test_shared_attention_refuses_caches(over):
    c = _cache(**over[0])
    assert qb.lib().qzo_paged_attention_shared(16, 256, 2, 2, 4, C.addressof(c), 16, 4, 16, None, 1, 16, 16, 0.1, 16, 256, 256, 1 << 30, None) == over[1]


# ------------------------------------------------------------------ forks ----
def _fork(parents, lengths, tables, free, n_free, block, group_starts=()):
    n = len(parents)
    d = dict(lengths=_i32(lengths), tables=_i32(tables), free=_i32(free), state=_i32([n_free, 7, 7, 7]), copies=torch.full((n, 4), -9, dtype=torch.int32, device=DEV))
    starts = _i32(group_starts) if len(group_starts) else None
    shared = torch.full((len(group_starts) - 1,), -9, dtype=torch.int32, device=DEV) if len(group_starts) else None
    qb.qzo_cache_fork(_i32(parents), block, *d.values(), group_starts=starts, shared=shared)
    torch.cuda.synchronize()
    out = {k: v.cpu().numpy() for k, v in d.items()}
    out["shared"] = [] if shared is None else shared.tolist()
    return out


def _check_fork(parents, lengths, tables, free, n_free, block, group_starts=()):
    want, got = fork_reference(parents, lengths, tables, free, n_free, block, group_starts), _fork(parents, lengths, tables, free, n_free, block, group_starts)
    if not isinstance(want, dict):
        want = dict(lengths=lengths, tables=tables, free=free, state=[n_free, 0, want, 0], copies=[], shared=got["shared"])
    assert list(got["lengths"]) == list(want["lengths"]) and (got["tables"] == want["tables"]).all() and (got["free"] == want["free"]).all()
    assert list(got["state"]) == want["state"] and got["shared"] == want["shared"]
    k = len(want["copies"])
    assert got["copies"][:k].tolist() == want["copies"] and (got["copies"][k:] == -9).all()
    return want


def _forest(lengths, block, most, spare, seed, alike=()):
    """Tables of sequences; in every range of `alike` they share the blocks that the shortest one has in full."""
    rng = np.random.default_rng(seed)
    need = [-(-x // block) for x in lengths]
    ids = rng.permutation(sum(need) + spare).astype(np.int32)
    tables, at = np.full((len(lengths), most), -5, dtype=np.int32), 0
    for i, k in enumerate(need):
        tables[i, :k] = ids[at:at + k]
        at += k
    free = np.full(len(ids), -6, dtype=np.int32)
    unused = list(ids[at:])
    for a, b in alike:
        k = min(lengths[a:b]) // block
        for i in range(a + 1, b):
            unused += list(tables[i, :k])
            tables[i, :k] = tables[a, :k]
    free[:len(unused)] = unused
    return tables, free, len(unused)


@gpu
@pytest.mark.parametrize("parents", [[0, 1, 2, 3], [0, 0, 0, 0], [3, 3, 3, 3], [3, 2, 1, 0], [1, 0, 0, -1], [-1, -1, -1, -1], [2, 2, 0, 0], [-1, 3, -1, 3], [1, 2, 3, 0]])
@pytest.mark.parametrize("lengths", [[40, 40, 40, 40], [48, 32, 1, 0], [16, 33, 100, 64], [0, 0, 0, 0], [5, 5, 5, 5]])
def test_fork(parents, lengths):
    tables, free, n_free = _forest(lengths, 16, 9, 5, 1)
    _check_fork(parents, lengths, tables, free, n_free, 16, [0, 4])
    tables, free, n_free = _forest(lengths, 16, 7, 3, 2, [(0, 2), (2, 4)])
    _check_fork(parents, lengths, tables, free, n_free, 16, [0, 2, 4])
    _check_fork(parents, lengths, tables, free, n_free, 16)


@gpu
@pytest.mark.parametrize("n,width,block,longest,seed", [(1, 1, 16, 50, 0), (6, 3, 32, 400, 1), (65, 5, 16, 90, 2), (300, 4, 64, 3000, 3), (1100, 11, 16, 700, 4), (8192, 64, 16, 33, 5),
                                                        (7, 7, 16, 20000, 6), (40, 40, 256, 9000, 7)])
def test_fork_again_and_again(n, width, block, longest, seed):
    rng = np.random.default_rng(seed)
    base = [int(x) for x in rng.integers(0, longest + 1, n // width + 1)]
    lengths = [base[i // width] + int(rng.integers(0, 40)) for i in range(n)]
    starts = list(range(0, n, width)) + [n]
    tables, free, n_free = _forest(lengths, block, -(-(longest + 40) // block) + 1, n, seed, list(zip(starts[:-1], starts[1:])))
    for turn in range(3):
        parents = [int(rng.integers(starts[i // width], min(n, starts[i // width] + width))) if rng.random() < 0.8 else i if rng.random() < 0.7 else -1 for i in range(n)]
        want = _check_fork(parents, lengths, tables, free, n_free, block, starts)
        assert want["state"][2] == 0
        lengths, tables, free, n_free = want["lengths"], want["tables"], want["free"], want["state"][0]


@gpu
@pytest.mark.parametrize("parents,lengths,n_free,status", [
    ([0, 2], [5, 5], 1, qb.QZO_ERR_ARG), ([0, 0], [5, -1], 1, qb.QZO_ERR_ARG), ([0, 0], [5, 5], -1, qb.QZO_ERR_ARG), ([0, 0], [5, 5], 99, qb.QZO_ERR_ARG),
    ([0, 0], [5, 65], 1, qb.QZO_ERR_SHAPE), ([0, 1], [5, 5], 0, 0), ([0, 0], [5, 0], 0, qb.QZO_ERR_WORKSPACE), ([0, 0], [5, 5], 0, 0), ([-1, -1], [5, 5], 3, qb.QZO_ERR_ARG)])
def test_fork_that_cannot_be_made_changes_nothing(parents, lengths, n_free, status):
    tables = np.array([[0, 1, 2, 3], [2, 3, 4, 5]], dtype=np.int32)
    free = np.array([1, 3, 4, 0], dtype=np.int32)
    want = fork_reference(parents, lengths, tables, free, n_free, 16)
    assert (status == 0) == isinstance(want, dict) and (status == 0 or want == status)
    _check_fork(parents, lengths, tables, free, n_free, 16)
    tables, free, n_free = _forest([20, 20], 16, 4, 3, 1)         # and nothing is left behind in the scratch
    for _ in range(2):
        _check_fork([1, 1], [20, 20], tables, free, n_free, 16, [0, 2])


@gpu
def test_fork_with_blocks_outside_the_pool():
    lengths, parents = [40, 40, 33, 20], [0, 0, 3, 3]
    tables, free, n_free = _forest(lengths, 16, 4, 4, 3)
    tables[1, 0], tables[2, 1], tables[3, 0] = len(free), -1, 1 << 30
    _check_fork(parents, lengths, tables, free, n_free, 16, [0, 2, 4])


@gpu
def test_group_starts_outside_the_sequences():
    lengths = [64, 64, 64]
    tables, free, n_free = _forest(lengths, 16, 4, 4, 3, [(0, 3)])
    got = _fork([0, 1, 2], lengths, tables, free, n_free, 16, [-5, 2, 2, 99])
    assert got["shared"] == [64, 0, 64]


# ------------------------------------------------------------------ compaction, copies ----
@gpu
@pytest.mark.parametrize("lengths,block,pool,alike", [
    ([0], 16, 1, ()), ([1], 16, 1, ()), ([16], 16, 5, ()), ([40, 0, 33], 16, 50, ()), ([100, 100, 90, 90], 32, 23, [(0, 2), (2, 4)]), ([2000] * 30, 16, 9000, [(0, 30)]),
    ([300] * 200, 16, 3801, ()), ([17] * 5000, 32, 40000, ()), ([30000], 16, 2048 * 16, ())])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(lengths, block, pool, alike, in_place):
    need = sum(-(-x // block) for x in lengths)
    tables, _, _ = _forest(lengths, block, max(1, max(-(-x // block) for x in lengths)) + 1, max(0, pool - need), 5, alike)
    pool = max(pool, need)
    for _ in range(2):
        t, free, state = _i32(tables), torch.full((pool,), -7, dtype=torch.int32, device=DEV), _i32([3, 3, 3, 3])
        new, copies = t if in_place else torch.full_like(t, -8), torch.full((max(1, pool // 2), 4), -9, dtype=torch.int32, device=DEV)
        qb.qzo_cache_compact(block, _i32(lengths), t, free, new, state, copies)
        held = sorted({int(b) for i, x in enumerate(lengths) for b in tables[i, :-(-x // block)]})
        k = len(held)
        far, holes = [b for b in held if b >= k], sorted(set(range(k)) - set(held))
        to = dict(zip(far, holes))
        want = tables.copy() if in_place else np.full_like(tables, -8)
        for i, x in enumerate(lengths):
            want[i, :-(-x // block)] = [to.get(int(b), int(b)) for b in tables[i, :-(-x // block)]]
        assert (new.cpu().numpy() == want).all() and (in_place or (t.cpu().numpy() == tables).all())
        assert state.tolist() == [pool - k, 0, 0, len(far)]
        assert free.tolist() == list(range(pool - 1, k - 1, -1)) + [-7] * k
        assert copies[:len(far)].tolist() == [[b, to[b], block, 0] for b in far] and (copies[len(far):] == -9).all()


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("layers,heads,block,dh", [(1, 1, 16, 64), (3, 5, 32, 128), (2, 40, 256, 64), (5, 2, 128, 128)])
def test_copy(layers, heads, block, dh, e4m3):
    rng = np.random.default_rng(1)
    pool = 23
    k, v = (torch.randint(-2**31, 2**31 - 1, (layers, pool, heads, block, dh // (4 if e4m3 else 2)), dtype=torch.int32, device=DEV).view(torch.float8_e4m3fn if e4m3 else torch.bfloat16)
            for _ in range(2))
    cache = qb.make_cache(k[0], v[0])
    ids = rng.permutation(pool)
    entries = [[int(ids[2 * i]), int(ids[2 * i + 1]), int(t), 0] for i, t in enumerate([1, block, block - 1, 3, 0, block + 9, 7])]
    entries += [[int(ids[20]), int(ids[20]), 5, 0], [-1, int(ids[21]), 5, 0], [int(ids[21]), pool, 5, 0], [int(ids[20]), int(ids[21]), -3, 0]]
    for count in (None, 0, 3, 99, -4):
        want = [x.view(torch.int16 if not e4m3 else torch.uint8).clone() for x in (k, v)]
        n = len(entries) if count is None else max(0, min(count, len(entries)))
        for a, b, t, _ in entries[:n]:
            if 0 <= a < pool and 0 <= b < pool and a != b and t > 0:
                for x in want:
                    x[:, b, :, :min(t, block)] = x[:, a, :, :min(t, block)].clone()
        qb.qzo_cache_copy(cache, _i32(entries), layers=layers, count=None if count is None else _i32([5, 5, 5, count]))
        for x, y in zip((k, v), want):
            assert torch.equal(x.view(y.dtype), y)


@gpu
def test_copy_beyond_32_bits():
    block, heads, dh, n = 64, 16, 128, 20000                # 5.2 GB a pool
    k, v = (torch.zeros(1, n, heads, block, dh, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[0, n - 1], v[0, n - 1] = 1.5, 2.5
    qb.qzo_cache_copy(qb.make_cache(k[0], v[0]), _i32([[n - 1, n - 3, 20, 0], [n - 1, 2, 64, 0]]))
    for x, y in ((k, 1.5), (v, 2.5)):
        assert (x[0, n - 3, :, :20] == y).all() and (x[0, n - 3, :, 20:] == 0).all() and (x[0, 2] == y).all() and (x[0, n - 2] == 0).all() and (x[0, 3:9] == 0).all()


# ------------------------------------------------------------------ the next beams ----
def _select(logits, width, scores, counts, ended, history, end, alpha):
    rows = logits.shape[0]
    d = dict(scores=torch.tensor(scores, dtype=torch.float32, device=DEV), counts=_i32(counts), ended=_i32(ended),
             history=_i32(history) if history.shape[1] else None, **{x: torch.full((rows,), -9, dtype=torch.int32, device=DEV) for x in ("parents", "chosen", "tokens", "added")})
    qb.qzo_beam_select(logits, width, *d.values(), end_token=end, length_penalty=alpha)
    return {k: v.cpu().numpy() if v is not None else history for k, v in d.items()}


def _check_select(logits, width, scores, counts, ended, history, end, alpha):
    want, gap = select_reference(logits.float().cpu().numpy().astype(np.float64), width, scores, counts, ended, history, end, alpha)
    # a row's sum is off by a few 2^-24 of it (each term's exponential by two, rescalings by one each): keys further apart than that are in order
    assert gap > 16 * 2.0 ** -24
    got = _select(logits, width, scores, counts, ended, history, end, alpha)
    for name in ("counts", "ended", "parents", "chosen", "added", "tokens"):
        assert list(got[name]) == list(want[name]), name
    assert (got["history"] == want["history"]).all()
    w = np.array(want["scores"])
    assert (np.isfinite(got["scores"]) == np.isfinite(w)).all()
    fin = np.isfinite(w)
    assert (np.abs(got["scores"][fin] - w[fin]) <= 2.0 ** -24 * np.abs(w[fin]) + 16 * 2.0 ** -24).all()
    return got


def _beams(groups, width, vocab, columns, seed, spread=2.0):
    rng = np.random.default_rng(seed)
    rows = groups * width
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    logits = (torch.randn(rows, vocab, generator=gen, device=DEV) * spread).to(torch.bfloat16)
    counts = [int(x) for x in rng.integers(0, columns + 1, rows)]
    scores = [float(np.float32(-3.0 * rng.random() * (1 + 0.1 * c))) for c in counts]
    history = rng.integers(0, vocab, (rows, columns)).astype(np.int32)
    return logits, scores, counts, history


@gpu
@pytest.mark.parametrize("alpha", [0.0, 0.7])
@pytest.mark.parametrize("groups,width,vocab,columns,seed", [
    (1, 1, 1, 0, 0), (1, 1, 50, 3, 1), (1, 4, 32000, 20, 2), (3, 5, 997, 7, 3), (2, 64, 300, 100, 4), (40, 3, 5001, 2, 5), (1, 8, 70000, 1, 6), (5, 33, 131, 11, 7),
    (1, 64, 1 << 20, 9, 8), (300, 2, 1023, 400, 9), (2, 7, 3, 4, 10)])
def test_select(groups, width, vocab, columns, seed, alpha):
    logits, scores, counts, history = _beams(groups, width, vocab, columns, seed)
    rows = groups * width
    ended = [int(i % 7 == 3) for i in range(rows)]
    scores = [-math.inf if i % 11 == 5 else s for i, s in enumerate(scores)]
    _check_select(logits, width, scores, counts, ended, history, vocab // 2, alpha)
    _check_select(logits, width, scores, counts, [0] * rows, history, -1, alpha)


@gpu
def test_select_at_the_start():
    """One beam of every prompt is there; the next ones all come from it."""
    logits, _, _, history = _beams(4, 6, 1000, 5, 3)
    scores = [0.0 if i % 6 == 0 else -math.inf for i in range(24)]
    logits[1::6] = math.nan                       # rows that are no beams are not looked at
    got = _check_select(logits, 6, scores, [0] * 24, [0] * 24, history, 7, 0.0)
    assert list(got["parents"]) == [i // 6 * 6 for i in range(24)]


@gpu
@pytest.mark.parametrize("vocab", [9, 1000, 40000])
def test_select_ties_go_to_the_lower_beam_and_token(vocab):
    logits = torch.zeros(6, vocab, dtype=torch.bfloat16, device=DEV)
    logits[:, ::2] = -0.0
    got = _check_select(logits, 3, [-1.0] * 6, [2] * 6, [0] * 6, np.zeros((6, 4), np.int32), -1, 0.0)
    assert list(got["chosen"]) == [0, 1, 2] * 2 and list(got["parents"]) == [0, 0, 0, 3, 3, 3]
    logits[1, vocab - 1] = logits[4, 5] = 2.0      # equal rows again, but for one token
    logits[0, vocab - 1] = logits[3, 5] = 2.0
    got = _check_select(logits, 3, [-1.0] * 6, [2] * 6, [0] * 6, np.zeros((6, 4), np.int32), -1, 0.0)
    assert list(got["parents"][:2]) == [0, 1] and list(got["chosen"][:2]) == [vocab - 1, vocab - 1] and list(got["chosen"][3:5]) == [5, 5]


@gpu
def test_select_leaves_out_what_is_not_finite():
    logits, scores, counts, history = _beams(3, 4, 3000, 6, 5)
    logits[:, ::3], logits[:, 1::3] = -math.inf, math.nan
    logits[2], logits[5, 2::3] = math.inf, math.inf
    logits[4:8] = -math.inf
    logits[4, 17], logits[6, 5] = 3.0, -200.0      # a prompt with two candidates for four beams
    got = _check_select(logits, 4, scores, counts, [0] * 12, history, 17, 0.0)
    assert sorted(got["chosen"][4:8]) == [-1, -1, 5, 17]
    got = _check_select(torch.full_like(logits, -math.inf), 4, scores, counts, [0, 0, 1, 0] * 3, history, 17, 0.0)
    assert list(got["chosen"]) == [17, -1, -1, -1] * 3


@gpu
@pytest.mark.parametrize("spread", [1e-3, 30.0, 1e4, 1e37])
def test_select_of_flat_and_steep_logits(spread):
    logits, scores, counts, history = _beams(2, 4, 5000, 6, 6, spread)
    _check_select(logits, 4, scores, counts, [0] * 8, history, 3, 0.5)


@gpu
@pytest.mark.parametrize("vocab,skip", [(1001, 0), (1001, 3), (8192, 5), (513, 1), (17, 7)])
def test_select_of_strided_rows(vocab, skip):
    """Rows at any multiple of two bytes, NaN between them."""
    logits, scores, counts, history = _beams(3, 3, vocab, 4, 7)
    wide = torch.full((9, vocab + 13), math.nan, dtype=torch.bfloat16, device=DEV)
    wide[:, skip:skip + vocab] = logits
    got = _check_select(wide[:, skip:skip + vocab], 3, scores, counts, [0] * 9, history, 2, 0.0)
    assert list(got["chosen"]) == list(_select(logits, 3, scores, counts, [0] * 9, history, 2, 0.0)["chosen"])


@gpu
def test_select_with_large_and_negative_counts():
    logits, scores, counts, history = _beams(2, 3, 500, 5, 8)
    counts = [3, 900, -4, 5, 2, 4]                  # longer than the history: no longer recorded
    _check_select(logits, 3, scores, counts, [0, 0, 0, 0, 1, 0], history, 2, 1.0)


@gpu
def test_select_sees_all_of_a_falling_row():
    """Every logit below the one before: the first tile has all the best; rising: every tile has better ones."""
    x = torch.arange(60000, 0, -1, device=DEV).float().mul(2.0 ** -12).to(torch.bfloat16)
    for row in (x, x.flip(0)):
        _check_select(row.repeat(5, 1).contiguous() * torch.tensor([1.0, 0.5, 0.25, 2.0, 1.0], device=DEV, dtype=torch.bfloat16)[:, None], 5, [-1.0, -2.0, -3.0, -4.0, -1.5], [1] * 5, [0] * 5,
                      np.zeros((5, 3), np.int32), -1, 0.0)


# ------------------------------------------------------------------ attention behind what is shared ----
def _attend(groups, shared, own, H, Hk, dh, block, news=None, e4m3=False, seed=0, spread=2.0, dead=(), claim=None, extra=3):
    """groups: how many sequences each has; shared: what they have in common, own: each one's tokens behind that, news: of them the new ones (None: one, without
    starts).  dead: sequences of length 0.  claim: what is passed as shared (default: all of it)."""
    rng, gen = np.random.default_rng(seed), torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n = sum(groups)
    starts_g = [0] + list(np.cumsum(groups))
    group = [g for g, k in enumerate(groups) for _ in range(k)]
    lengths = [0 if i in dead else shared[group[i]] + own[i] for i in range(n)]
    most = max(1, max(-(-x // block) for x in lengths)) + 1
    need = [[-(-x // block)] for x in lengths]
    pool = sum(x[0] for x in need) + sum(x // block for x in shared) + extra
    ids = list(rng.permutation(pool))
    tables = np.full((n, most), -1, np.int32)
    for g in range(len(groups)):
        k = shared[g] // block
        common = [ids.pop() for _ in range(k)] if groups[g] else []
        for i in range(starts_g[g], starts_g[g + 1]):
            if lengths[i]:
                tables[i, :need[i][0]] = common + [ids.pop() for _ in range(need[i][0] - k)]
    shape = (pool, Hk, block, dh)
    k, v = (torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    # the shared part's last, open block: the same in everyone's own
    for g in range(len(groups)):
        live = [i for i in range(starts_g[g], starts_g[g + 1]) if lengths[i]]
        r, at = shared[g] % block, shared[g] // block
        for i in live[1:]:
            if r:
                for x in (k, v):
                    x[tables[i, at], :, :r] = x[tables[live[0], at], :, :r]
    scales = [None, None]
    kk, vv = k, v
    if e4m3:
        scales = [torch.rand(Hk, generator=gen, device=DEV) * 0.2 + 0.05 for _ in range(2)]
        kk, vv = ((x.float() * 4).to(torch.float8_e4m3fn) for x in (k, v))
    new = [1] * n if news is None else [0 if i in dead else news[i] for i in range(n)]
    starts = [0] + list(np.cumsum(new))
    q = (torch.randn(starts[-1], H * dh, generator=gen, device=DEV) * spread).to(torch.bfloat16)
    return dict(q=q, k=kk, v=vv, scales=scales, tables=_i32(tables), lengths=_i32(lengths), starts=None if news is None else _i32(starts), starts_list=starts, group_starts=_i32(starts_g),
                shared=_i32(shared if claim is None else claim), H=H, dh=dh, scale=1.0 / math.sqrt(dh), pad=2)


def _shared_call(d, **more):
    cache = qb.make_cache(d["k"], d["v"], *d["scales"])
    rows, width = d["q"].shape
    q = torch.full((rows + d["pad"], width), math.nan, dtype=torch.bfloat16, device=DEV) if d["starts"] is not None else d["q"]
    q[:rows] = d["q"]
    out = torch.full_like(q, 77.0)
    qb.qzo_paged_attention_shared(q, cache, d["tables"], d["lengths"], d["group_starts"], d["shared"], out, d["scale"], starts=d["starts"], **more)
    assert (out[rows:] == 77.0).all()
    return out[:rows]


def _check_shared(d, parts=1):
    got = _shared_call(d)
    pools = []
    for x, s in zip((d["k"], d["v"]), d["scales"]):
        pools.append(x.double() if s is None else x.float().double() * s.double()[:, None, None])
    q = d["q"].double().view(-1, d["H"], d["dh"])
    want, mag, mac = attention_reference(q, *pools, d["tables"], d["lengths"].tolist(), d["starts_list"], d["scale"])
    # joining two shares takes a few more fp32 steps: an exponential, two products and a sum each
    tol = attention_tolerance(want, mag, mac, d["dh"]) + 16 * 2.0 ** -24 * mag
    err = (got.double().view_as(want) - want).abs()
    assert (err <= tol).all(), (err / tol).max()
    return got


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("groups,shared,own,H,Hk,dh,block", [
    ([4], [64], [1, 2, 17, 40], 4, 4, 128, 16), ([4], [500], [1, 20, 3, 16], 32, 32, 128, 16), ([2, 3], [100, 33], [5, 1, 9, 16, 50], 8, 2, 64, 32),
    ([1, 5, 0, 2], [40, 300, 90, 0], [9, 3, 4, 5, 6, 7, 8, 100], 6, 2, 128, 64), ([64], [700], list(range(1, 65)), 8, 1, 64, 16), ([8] * 16, [i * 37 for i in range(16)], [1 + i % 23 for i in range(128)], 4, 4, 64, 16),
    ([3] * 3, [15, 16, 17], [1] * 9, 5, 5, 128, 128), ([100], [2000], [1 + i * 3 for i in range(100)], 16, 2, 128, 32), ([2], [9000], [700, 1], 2, 2, 128, 16)])
def test_attention_behind_what_is_shared(groups, shared, own, H, Hk, dh, block, e4m3):
    _check_shared(_attend(groups, shared, own, H, Hk, dh, block, e4m3=e4m3, seed=len(own)))


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("groups,shared,own,news,H,Hk,dh,block", [
    ([3], [48], [5, 6, 7], [5, 2, 7], 4, 2, 64, 16), ([12], [300], [9] * 12, [9] * 12, 10, 2, 64, 16), ([4, 4], [1000, 90], [40] * 8, [40] * 8, 4, 4, 128, 32),
    ([2], [33], [200, 190], [200, 100], 8, 2, 128, 64), ([5, 3], [640, 64], [30, 1, 2, 3, 25, 90, 80, 70], [30, 1, 2, 0, 25, 90, 1, 70], 16, 2, 128, 16)])
def test_several_new_tokens_behind_what_is_shared(groups, shared, own, news, H, Hk, dh, block, e4m3):
    _check_shared(_attend(groups, shared, own, H, Hk, dh, block, news=news, e4m3=e4m3, seed=len(own)))


@gpu
@pytest.mark.parametrize("news", [None, [2, 2, 2, 2, 3]])
def test_sequences_that_have_ended(news):
    """Length 0, first of its group, too; without starts their rows become zero."""
    for dead in ((0,), (2, 4), (1, 2, 3, 4), (0, 1, 2, 3, 4)):
        d = _attend([5], [100], [5, 4, 3, 7, 9], 4, 2, 128, 16, news=news, dead=dead, seed=3)
        got = _check_shared(d)
        if news is None:
            assert (got[list(dead)] == 0).all()


@gpu
@pytest.mark.parametrize("claim", [[0, 0], [-7, 1 << 30], [20, 37], [64, 31], [90, 1]])
def test_what_is_claimed_to_be_shared(claim):
    """Less than is: any number of tokens.  More than a sequence has behind its new tokens: it reads its own."""
    shared = [max(0, x) for x in claim]
    d = _attend([3, 2], [96, 64], [7, 3, 20, 9, 1], 4, 2, 64, 32, seed=4, claim=claim)
    if any(x > y for x, y in zip(shared, [96, 64])):
        d["shared"] = _i32([claim[0], 1 << 30])      # beyond all lengths
    _check_shared(d)


@gpu
def test_sequences_in_no_group():
    d = _attend([2, 3, 2], [50, 64, 80], [5, 3, 20, 9, 1, 6, 7], 4, 2, 64, 16, seed=5)
    d["group_starts"], d["shared"] = _i32([2, 5]), _i32([64])
    _check_shared(d)
    d["group_starts"], d["shared"] = _i32([-3, 2, 2, 5, 1000]), _i32([50, 9, 64, 80])
    _check_shared(d)


@gpu
def test_shared_equals_unshared_bits_where_nothing_is():
    d = _attend([3, 3], [0, 0], [300, 200, 4, 700, 1, 64], 8, 2, 128, 16, seed=6)
    cache = qb.make_cache(d["k"], d["v"])
    out = torch.zeros_like(d["q"])
    qb.qzo_paged_attention(d["q"], cache, d["tables"], d["lengths"], out, d["scale"])
    assert (_shared_call(d).float() - out.float()).abs().max() <= 2.0 ** -7 * out.float().abs().max()


@gpu
def test_unseen_positions_of_shared_blocks_hold_anything():
    """Behind every sequence's last token, in blocks that nobody holds, in rows that are padding."""
    for news in (None, [3, 1, 5, 2]):
        d = _attend([2, 2], [48, 96], [5, 9, 20, 3], 4, 2, 128, 32, news=news, seed=7)
        used = torch.zeros(d["k"].shape[0], 32, dtype=torch.bool, device=DEV)
        for i, x in enumerate(d["lengths"].tolist()):
            at = torch.arange(x, device=DEV)
            used[d["tables"][i, at // 32].long(), at % 32] = True
        for x in (d["k"], d["v"]):
            y = torch.where(used[:, None, :, None], x, torch.tensor(math.nan, dtype=torch.bfloat16, device=DEV))
            x.copy_(y)
        want_k, want_v = (torch.where(used[:, None, :, None], x, torch.zeros_like(x)) for x in (d["k"], d["v"]))
        got = _shared_call(d)
        d["k"], d["v"] = want_k, want_v
        assert torch.equal(got, _check_shared(d))


@gpu
def test_a_query_of_nan_stays_alone():
    d = _attend([4], [200], [5, 9, 20, 3], 4, 4, 128, 16, seed=8)
    want = _shared_call(d)
    d["q"][2, :128] = math.nan
    got = _shared_call(d)
    assert got[2, :128].isnan().all()
    got[2, :128] = want[2, :128]
    assert torch.equal(got, want)


@gpu
def test_more_items_than_a_launch_has_room_for():
    n, groups = 7000, 2000
    d = _attend([3] * groups + [1] * (n - 3 * groups), [32] * groups + [0] * (n - 3 * groups), [1 + i % 9 for i in range(n)], 1, 1, 64, 16, seed=9)
    d["group_starts"], d["shared"] = _i32([3 * i for i in range(groups + 1)]), _i32([32] * groups)
    _check_shared(d)


@gpu
def test_strided_rows():
    d = _attend([3, 2], [96, 64], [7, 3, 20, 9, 1], 4, 2, 64, 32, seed=4)
    want = _shared_call(d)
    wide, out = torch.zeros(5, 3 * 256, dtype=torch.bfloat16, device=DEV), torch.full((5, 512), 9.0, dtype=torch.bfloat16, device=DEV)
    wide[:, 256:512] = d["q"]
    qb.qzo_paged_attention_shared(wide[:, 256:512], qb.make_cache(d["k"], d["v"]), d["tables"], d["lengths"], d["group_starts"], d["shared"], out[:, :256], d["scale"])
    assert torch.equal(out[:, :256], want) and (out[:, 256:] == 9.0).all()


@gpu
def test_the_same_call_gives_the_same_bits():
    for seed, (groups, shared, H, Hk, dh) in enumerate([([8] * 4, [900, 30, 444, 0], 8, 8, 128), ([40], [3000], 16, 2, 64)]):
        d = _attend(groups, shared, [1 + 5 * i for i in range(sum(groups))], H, Hk, dh, 16, seed=seed)
        first = _shared_call(d)
        for _ in range(5):
            assert torch.equal(_shared_call(d), first)


# ------------------------------------------------------------------ with a model ----
@gpu
@pytest.mark.parametrize("name,e4m3,width,alpha,end", [("tiny", False, 4, 0.0, -1), ("wide_heads", False, 3, 0.6, 5), ("tiny_opt", True, 5, 1.0, 7), ("tiny", False, 1, 0.0, -1)])
def test_beams_of_a_model(name, e4m3, width, alpha, end):
    """Every step's beams are those of the definition, given its logits; the logits are those of the model over prompt and history."""
    m = _model(name, "int4")
    rng = torch.Generator().manual_seed(4)
    texts = [torch.randint(0, m.shape["vocab"], (n,), generator=rng, dtype=torch.int32).to(DEV) for n in (61, 16, 33)]
    new = 20
    b = Beams(m, 3, width, n_blocks=60, max_new=new, end_token=end, length_penalty=alpha, block=16, max_blocks=9, e4m3=e4m3)
    b.start(torch.cat(texts), _i32([t.numel() for t in texts]))
    a, n = b.answers, 3 * width
    for turn in range(1, new):
        before = {k: getattr(b, k).cpu().numpy().copy() for k in ("scores", "counts", "ended", "history")}
        on = b.added.tolist()
        # a beam's last token is not in the cache yet
        assert a.lengths.tolist() == [texts[i // width].numel() + before["counts"][i] - 1 for i in range(n)]
        b.step()
        logits = a.logits.clone()
        for i in range(n):
            if on[i] and turn % 4 == 1:
                text = torch.cat([texts[i // width], _i32(before["history"][i, :before["counts"][i]])])
                want = _logits(m, text)
                assert _far(logits[i], want[-1]) <= max(0.1 if e4m3 else 2e-2, 2 * _apart(m, text, want)), (turn, i)
        want, gap = select_reference(logits.float().cpu().numpy().astype(np.float64), width, before["scores"], [int(x) for x in before["counts"]], before["ended"], before["history"], end, alpha)
        assert gap > 16 * 2.0 ** -24
        for k in ("counts", "ended", "parents", "chosen", "added", "tokens"):
            assert getattr(b, k).tolist() == list(want[k]), k
        assert (b.history.cpu().numpy() == want["history"]).all() and int(b.failed) == 0
        _check_cache(a)
    assert (a.shared >= torch.tensor([48, 16, 32], device=DEV)).all()       # the prompts' full blocks at least
    history, counts, scores = Beams(m, 3, width, n_blocks=60, max_new=new, end_token=end, length_penalty=alpha, block=16, max_blocks=9, e4m3=e4m3).search(
        torch.cat(texts), _i32([t.numel() for t in texts]), look_every=5)
    assert torch.equal(counts.view(-1), b.counts) and torch.equal(scores.view(-1), b.scores)
    for i in range(n):
        assert history.view(n, -1)[i, :counts.view(-1)[i]].tolist() == b.history[i, :b.counts[i]].tolist()


def _check_cache(a):
    """Every block is held or free, once; open blocks are one sequence's."""
    lengths, tables, free = a.lengths.tolist(), a.tables.cpu().numpy(), a.free[:int(a.state[0])].tolist()
    held = [list(tables[i, :-(-x // a.block)]) for i, x in enumerate(lengths)]
    all_held = {b for row in held for b in row}
    assert len(free) == len(set(free)) and not all_held & set(free) and len(all_held) + len(free) == a.free.numel()
    opened = [row[-1] for row, x in zip(held, lengths) if x % a.block]
    assert len(opened) == len(set(opened)) and not any(b in row[:-1] for b in opened for row in held)


@gpu
def test_captured_beams_replay():
    """A step captured into a graph writes the same beams as eager ones, the program's own work in between."""
    m = _model("tiny", "int4")
    tokens, lengths = torch.arange(70, dtype=torch.int32, device=DEV) * 11, _i32([50, 20])
    seen = []
    for captured in (False, True):
        b = Beams(m, 2, 4, n_blocks=80, max_new=40, end_token=3, block=16, max_blocks=9)
        for _ in range(2):                         # a second search in the same place
            b.start(tokens, lengths)
            b.step()
            torch.cuda.synchronize()
            if captured:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    b.step()
            found = []
            for i in range(25):
                g.replay() if captured else b.step()
                torch.cuda.synchronize()
                m.forward_loss(tokens.view(1, -1)[:, :40].contiguous(), 1, 1e-3, 1)
                found += [b.history.clone(), b.scores.clone(), b.answers.lengths.clone()]
            assert int(b.failed) == 0
            _check_cache(b.answers)
            seen.append(found)
    for other in seen[1:]:
        assert all(torch.equal(x, y) for x, y in zip(seen[0], other))


@gpu
def test_candidates_behind_a_prompt():
    """A prompt once, candidates of several tokens behind it: the same logits as with a copy of the prompt for each."""
    m = _model("tiny", "int4")
    rng = torch.Generator().manual_seed(5)
    prompt = torch.randint(0, 1024, (75,), generator=rng, dtype=torch.int32).to(DEV)
    parts = [torch.randint(0, 1024, (k,), generator=rng, dtype=torch.int32).to(DEV) for k in (5, 1, 9, 30)]
    a = Answers(m, n_seq=4, n_blocks=30, block=16, width=4)
    a.add(prompt, _i32([75, 0, 0, 0]))
    a.fork(_i32([0, 0, 0, 0]))
    assert a.shared.tolist() == [64] and a.state.tolist() == [30 - 5 - 3, 0, 0, 3]
    got = a.add(torch.cat(parts), _i32([p.numel() for p in parts])).clone()
    for i, p in enumerate(parts):
        text = torch.cat([prompt, p])
        want = _logits(m, text)
        assert _far(got[i], want[-1]) <= max(2e-2, 2 * _apart(m, text, want))
    _check_cache(a)
    a.add(torch.zeros(0, dtype=torch.int32, device=DEV), _i32([0, -1, -1, 0]))        # two end: what the others hold stays
    assert a.lengths.tolist() == [80, 0, 0, 105]
    _check_cache(a)
    a.add(torch.zeros(2, dtype=torch.int32, device=DEV), _i32([-1, 2, 0, -1]))
    assert a.lengths.tolist() == [0, 2, 0, 0] and a.shared.tolist() == [0]
    _check_cache(a)


@gpu
def test_pools_of_another_size():
    """Sequences are compacted into smaller pools, then larger ones, and go on as before."""
    m = _model("tiny", "int4")
    text = torch.randint(0, 1024, (120,), generator=torch.Generator().manual_seed(6), dtype=torch.int32).to(DEV)
    for width in (None, 2):
        runs = []
        for resized in (False, True):
            a = Answers(m, n_seq=4, n_blocks=40, block=16, max_blocks=9, width=width)
            a.add(text, _i32([40, 17, 50, 13]))
            a.fork(_i32([2, 1, 2, -1]))
            if resized:
                a.resize(12)
                assert a.k.shape[1] == a.free.numel() == 12
                _check_cache(a)
            out = [a.add(text[:3].contiguous(), _i32([1, 1, 1, 0])).clone()]
            if resized:
                with pytest.raises(ValueError):
                    a.resize(3)
                _check_cache(a)
                a.resize(100)
                _check_cache(a)
            out.append(a.add(text[:40].contiguous(), _i32([30, 1, 1, 8])).clone())
            assert a.state.tolist()[2] == 0
            runs.append(out)
        for x, y in zip(*runs):
            assert torch.equal(x, y)


@gpu
def test_a_fork_without_blocks_for_it():
    m = _model("tiny", "int4")
    a = Answers(m, n_seq=3, n_blocks=3, block=16, width=3)
    a.add(torch.zeros(40, dtype=torch.int32, device=DEV), _i32([40, 0, 0]))
    before = [x.clone() for x in (a.k.view(torch.int16), a.v.view(torch.int16), a.tables, a.lengths, a.free)]
    a.fork(_i32([0, 0, -1]))
    assert a.state.tolist() == [0, 0, qb.QZO_ERR_WORKSPACE, 0]
    assert all(torch.equal(x, y) for x, y in zip(before, (a.k.view(torch.int16), a.v.view(torch.int16), a.tables, a.lengths, a.free)))
    b = Beams(m, 1, 4, n_blocks=4, max_new=3, block=16)
    with pytest.raises(RuntimeError):
        b.search(torch.zeros(40, dtype=torch.int32, device=DEV), _i32([40]))


@gpu
def test_profile_of_an_answer_behind_what_is_shared():
    m = _model("tiny", "int4")
    a = Answers(m, n_seq=4, n_blocks=30, block=16, width=4)
    a.add(torch.arange(20, dtype=torch.int32, device=DEV), _i32([20, 0, 0, 0]))
    a.fork(_i32([0] * 4))
    qb.qzo_profile_begin(100)
    a._add(torch.arange(4, dtype=torch.int32, device=DEV), _i32([1] * 4))
    got = qb.qzo_profile_collect(qb.PROFILE_KINDS["attention"])
    assert got["launches"] == 2 and got["work"] == 0 and got["total_ms"] > 0


# ------------------------------------------------------------------ streams, scratch ----
@gpu
def test_forks_on_two_streams_at_once():
    """Scratch by stream: two pools of the same size, forked, selected and attended to at once."""
    lengths, parents, starts = [700] * 60, [i // 2 * 2 for i in range(60)], list(range(0, 61, 4))
    tables, free, n_free = _forest(lengths, 16, 45, 80, 1, [(i, i + 4) for i in range(0, 60, 4)])
    want = fork_reference(parents, lengths, tables, free, n_free, 16, starts)
    d = _attend([8] * 6, [400] * 6, [1 + i for i in range(48)], 4, 4, 128, 16, seed=2)
    out_want = _shared_call(d)
    logits, scores, counts, history = _beams(6, 8, 5000, 6, 2)
    sel_want = _select(logits, 8, scores, counts, [0] * 48, history, -1, 0.0)
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    torch.cuda.synchronize()
    for turn in range(6):
        for s in streams:
            with torch.cuda.stream(s):
                x = [_i32(lengths), _i32(tables), _i32(free), _i32([n_free, 0, 0, 0]), torch.zeros(60, 4, dtype=torch.int32, device=DEV)]
                qb.qzo_cache_fork(_i32(parents), 16, *x, group_starts=_i32(starts), shared=torch.zeros(15, dtype=torch.int32, device=DEV))
                o = torch.zeros_like(d["q"])
                qb.qzo_paged_attention_shared(d["q"], qb.make_cache(d["k"], d["v"]), d["tables"], d["lengths"], d["group_starts"], d["shared"], o, d["scale"])
                y = [torch.tensor(scores, device=DEV), _i32(counts), _i32([0] * 48), _i32(history)] + [torch.zeros(48, dtype=torch.int32, device=DEV) for _ in range(4)]
                qb.qzo_beam_select(logits, 8, *y)
                got.append((x, o, y))
    torch.cuda.synchronize()
    for x, o, y in got:
        assert x[0].tolist() == list(want["lengths"]) and (x[1].cpu().numpy() == want["tables"]).all() and (x[2].cpu().numpy() == want["free"]).all()
        assert x[3].tolist() == want["state"] and torch.equal(o, out_want) and (y[3].cpu().numpy() == sel_want["history"]).all()


@gpu
def test_captured_calls_need_scratch_of_their_own():
    logits, scores, counts, history = _beams(1, 2, 100, 2, 1)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    y = [torch.tensor(scores, device=DEV), _i32(counts), _i32([0] * 2), _i32(history)] + [torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        with pytest.raises(AssertionError):
            qb.qzo_beam_select(logits, 2, *y)
        torch.zeros(4, device=DEV).add_(1)


@gpu
def test_operands_elsewhere_are_refused():
    logits, scores, counts, history = _beams(1, 2, 100, 2, 1)
    good = [torch.tensor(scores, device=DEV), _i32(counts), _i32([0] * 2), _i32(history)] + [torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(4)]
    for i in range(len(good)):
        for bad in (good[i].cpu(), good[i].long()):
            with pytest.raises(AssertionError):
                qb.qzo_beam_select(logits, 2, *good[:i], bad, *good[i + 1:])
    with pytest.raises(AssertionError):
        qb.qzo_beam_select(logits.float(), 2, *good)
    with pytest.raises(qb.QzoError):
        qb.qzo_beam_select(logits, 2, *good, scratch=torch.zeros(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(AssertionError):
        qb.qzo_beam_select(logits, 2, *good, scratch=torch.zeros(1 << 20, dtype=torch.uint8))


# ------------------------------------------------------------------ common keys of many columns ----
@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("groups,shared,own,news,H,Hk,dh,block", [
    ([66], [16], [1] * 66, None, 1, 1, 128, 16), ([66], [48], [1] * 66, None, 1, 1, 64, 16), ([130], [64], [1 + i % 5 for i in range(130)], None, 2, 2, 128, 32),
    ([33], [1007], [3] * 33, None, 24, 3, 128, 64), ([9, 2, 40], [80, 2000, 333], [5] * 51, [5] * 51, 16, 4, 64, 16), ([3, 80], [5000, 64], [1] * 83, None, 8, 1, 128, 128),
    ([2] * 20, [100 + 61 * i for i in range(20)], [40] * 40, [40] * 40, 4, 2, 128, 16), ([300], [4000], [2] * 300, None, 4, 1, 64, 256)])
def test_common_keys_of_many_columns(groups, shared, own, news, H, Hk, dh, block, e4m3):
    _check_shared(_attend(groups, shared, own, H, Hk, dh, block, news=news, e4m3=e4m3, seed=sum(groups)))


@gpu
@pytest.mark.parametrize("n", [4, 40, 90])
@pytest.mark.parametrize("scale", [0.2, -0.2, 0.0, 3.0])
def test_scales_of_common_keys(n, scale):
    d = _attend([n], [90], [3] * n, 4, 2, 64, 16, seed=n)
    d["scale"] = scale
    _check_shared(d)


@gpu
@pytest.mark.parametrize("n", [4, 40, 90])
def test_absent_blocks_of_common_keys(n):
    d = _attend([n], [300], [20] * n, 4, 2, 128, 16, seed=n)
    d["tables"][:, 3], d["tables"][:, 17] = d["k"].shape[0] + 5, -1
    _check_shared(d)
    d["tables"][:, :18] = -7                        # all of what is common
    _check_shared(d)


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("n,dh", [(4, 128), (40, 64), (90, 128), (150, 64)])
def test_values_that_are_not_finite(n, dh, e4m3):
    """A common key that no row sees, by a score of -infinity, hides its value; one that is seen gives its NaN to its feature alone; a row of NaN stays alone."""
    d = _attend([n], [200], [5] * n, 2, 1, dh, 32, e4m3=e4m3, seed=n)
    want = _shared_call(d)
    at, p = d["tables"][0, 2].long(), 70 % 32       # position 70
    if not e4m3:
        k0, v0 = d["k"][at, :, p].clone(), d["v"][at, :, p].clone()
        d["q"].view(n, 2, dh)[..., 0] = d["q"].view(n, 2, dh)[..., 0].abs() + 0.25
        d["k"][at, :, p, 0] = -math.inf
        d["v"][at, :, p] = 0.0
        finite = _check_shared(d)
        d["v"][at, :, p] = math.nan
        assert (_shared_call(d).float() - finite.float()).abs().max() <= 2.0 ** -7 * finite.float().abs().max()
        d["v"][at, :, p, 1::2] = -math.inf
        assert (_shared_call(d).float() - finite.float()).abs().max() <= 2.0 ** -7 * finite.float().abs().max()
        d["k"][at, :, p], d["v"][at, :, p] = k0, v0
        want = _shared_call(d)
    d["v"].view(torch.uint8 if e4m3 else torch.int16)[at, :, p, 5] = 0x7f if e4m3 else 0x7fc0
    got = _shared_call(d).view(n, 2, dh)
    assert got[..., 5].isnan().all()
    rest = torch.arange(dh, device=DEV) != 5
    assert (got[..., rest].float() - want.view(n, 2, dh)[..., rest].float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
    d = _attend([n], [200], [5] * n, 2, 1, dh, 32, e4m3=e4m3, seed=n)
    want = _shared_call(d)
    d["q"][n // 2, 3] = math.nan
    got = _shared_call(d)
    assert got[n // 2, :dh].isnan().all()
    got[n // 2, :dh] = want[n // 2, :dh]
    assert torch.equal(got, want)


# ------------------------------------------------------------------ captured, long, out of order ----
@gpu
@pytest.mark.parametrize("n,longest", [(300, 90), (12, 700), (40, 7000)])
def test_captured_forks_replay(n, longest):
    """Few and many sequences: a captured fork and its copies, replayed on other parents with the program's own work in between."""
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in rng.integers(0, longest, n)]
    starts = list(range(0, n, 4)) + [n]
    tables, free, n_free = _forest(lengths, 16, -(-longest // 16) + 1, n, n, [(i, min(i + 3, n)) for i in range(0, n, 4)])
    kept = [_i32(lengths), _i32(tables), _i32(free), _i32([n_free, 0, 0, 0]), torch.full((n, 4), -9, dtype=torch.int32, device=DEV)]
    x, parents, shared = [t.clone() for t in kept], torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(len(starts) - 1, dtype=torch.int32, device=DEV)
    group_starts = _i32(starts)
    pool = torch.zeros(2, len(free), 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    filled = torch.randint(0, 30000, pool.shape, dtype=torch.int16, device=DEV).view(torch.bfloat16)
    cache = qb.make_cache(pool[0], pool[1])
    room = torch.zeros(qb.qzo_cache_fork_scratch_bytes(n, len(free), tables.shape[1]), dtype=torch.uint8, device=DEV)

    def step():
        for t, k in zip(x, kept):
            t.copy_(k)
        pool.copy_(filled)
        qb.qzo_cache_fork(parents, 16, *x, group_starts=group_starts, shared=shared, scratch=room)
        qb.qzo_cache_copy(cache, x[4], count=x[3])

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for turn in range(4):
        p = [int(i) for i in (rng.integers(-1, n, n) if turn % 2 else np.clip(np.arange(n) // 4 * 4 + rng.integers(0, 4, n), 0, n - 1))]
        parents.copy_(_i32(p))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = fork_reference(p, lengths, tables, free, n_free, 16, starts)
        assert isinstance(want, dict) and x[0].tolist() == list(want["lengths"]) and (x[1].cpu().numpy() == want["tables"]).all()
        assert (x[2].cpu().numpy() == want["free"]).all() and x[3].tolist() == want["state"] and shared.tolist() == want["shared"]
        assert x[4][:len(want["copies"])].tolist() == want["copies"]
        moved = filled.view(torch.int16).clone()
        for a, b, tokens, _ in want["copies"]:
            moved[:, b, :, :tokens] = moved[:, a, :, :tokens]
        assert torch.equal(pool.view(torch.int16), moved)
        assert _fork(p, lengths, tables, free, n_free, 16, starts)["state"].tolist() == want["state"]         # eager, by scratch of its own


@gpu
@pytest.mark.parametrize("n,dh,e4m3", [(4, 128, False), (40, 64, True), (90, 128, False)])
def test_captured_shared_attention_replays(n, dh, e4m3):
    """Queries and lengths that change between replays."""
    d, gen = _attend([n, n], [500, 90], [30] * (2 * n), 4, 2, dh, 16, e4m3=e4m3, seed=n), torch.Generator(device=DEV)
    cache = qb.make_cache(d["k"], d["v"], *d["scales"])
    room = torch.zeros(qb.qzo_paged_attention_shared_scratch_bytes(2 * n, 2 * n, 4, 2, dh), dtype=torch.uint8, device=DEV)
    out, side = torch.zeros_like(d["q"]), torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        qb.qzo_paged_attention_shared(d["q"], cache, d["tables"], d["lengths"], d["group_starts"], d["shared"], out, d["scale"], scratch=room)
    for turn in range(4):
        d["q"].copy_(torch.randn(d["q"].shape, generator=gen, device=DEV))
        d["lengths"].sub_(turn * 2 + 1)
        d["shared"].sub_(turn * 9)
        torch.cuda.synchronize()
        g.replay()
        other = _check_shared(d)
        torch.cuda.synchronize()
        assert torch.equal(out, other)


@gpu
def test_select_with_a_history_of_many_columns():
    """64 beams of 2^26 columns: columns times beams are beyond 32 bits."""
    columns = 1 << 26
    history = torch.empty(64, columns, dtype=torch.int32, device=DEV)
    torch.arange(columns, dtype=torch.int32, device=DEV, out=history[5])
    logits = torch.linspace(4.0, -4.0, 64, device=DEV).to(torch.bfloat16).repeat(64, 1)
    scores, counts = torch.full((64,), -math.inf, device=DEV), torch.zeros(64, dtype=torch.int32, device=DEV)
    scores[5], counts[5] = 0.0, columns - 1
    rest = [torch.zeros(64, dtype=torch.int32, device=DEV) for _ in range(5)]
    qb.qzo_beam_select(logits, 64, scores, counts, rest[0], history, *rest[1:])
    torch.cuda.synchronize()
    assert rest[1].tolist() == [5] * 64 and rest[2].tolist() == list(range(64)) and (counts == columns).all()
    assert history[:, -1].tolist() == list(range(64))
    for i in (0, 4, 5, 6, 63):
        assert torch.equal(history[i, :-1], torch.arange(columns - 1, dtype=torch.int32, device=DEV))


# ------------------------------------------------------------------ sequences that end and begin among those that share ----
def _refill(d, i, length, seed=0):
    """Sequence i of what _attend made, which has ended, begins again: `length` tokens, all of them new, in blocks that nobody holds."""
    gen, block = torch.Generator(device=DEV).manual_seed(seed), d["k"].shape[2]
    assert d["starts"] is not None and int(d["lengths"][i]) == 0
    n = -(-length // block)
    unused = sorted(set(range(d["k"].shape[0])) - set(d["tables"].flatten().tolist()))
    d["tables"] = torch.nn.functional.pad(d["tables"], (0, max(0, n - d["tables"].shape[1])), value=-1)
    d["tables"][i, :n] = _i32(unused[:n])
    d["lengths"][i] = length
    at, starts = d["starts_list"][i], d["starts_list"]
    q = torch.randn(length, d["q"].shape[1], generator=gen, device=DEV).to(torch.bfloat16)
    d["q"] = torch.cat([d["q"][:at], q, d["q"][at:]])
    d["starts_list"] = starts[:i + 1] + [x + length for x in starts[i + 1:]]
    d["starts"] = _i32(d["starts_list"])


@gpu
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("length", [1, 16, 20, 63, 64, 65, 100])
@pytest.mark.parametrize("n,H,Hk,dh", [(4, 4, 4, 128), (4, 4, 2, 64), (40, 4, 2, 128), (150, 1, 1, 64)])
def test_a_sequence_that_begins_among_those_that_share(n, H, Hk, dh, length, e4m3):
    """Its keys are not the group's, however many they are; first of its group, in the middle, and both."""
    for dead in ((0,), (n // 2,), (0, 1, n - 1)):
        d = _attend([n, 3], [64, 48], [12] * (n + 3), H, Hk, dh, 16, news=[1] * (n + 3), e4m3=e4m3, dead=dead, seed=n + length, extra=30)
        for i in dead:
            _refill(d, i, length, seed=i)
        _check_shared(d)


@gpu
@pytest.mark.parametrize("news", [False, True])
@pytest.mark.parametrize("n,H,Hk,dh", [(5, 4, 4, 128), (90, 4, 2, 64), (600, 1, 1, 64)])
def test_who_has_the_common_keys(n, H, Hk, dh, news):
    """They are read through the table of the first sequence that has them before its new tokens: what the others' tables name there does not matter."""
    for dead in ((), (0,), (0, 1, 3), tuple(range(n - 2))):
        d = _attend([n, 2], [64, 32], [12] * (n + 2), H, Hk, dh, 16, news=[1 + 2 * (i % 2) for i in range(n + 2)] if news else None, dead=dead, seed=n + len(dead))
        want = _check_shared(d)
        first = min(set(range(n)) - set(dead))
        for i in range(first + 1, n):
            d["tables"][i, :4] = -1
        assert torch.equal(_shared_call(d), want)


@gpu
@pytest.mark.parametrize("name,e4m3", [("tiny", False), ("wide_heads", False), ("tiny", True)])
@pytest.mark.parametrize("length", [20, 40, 100])
def test_a_new_prompt_beside_candidates(name, e4m3, length):
    """In the step in which the others go on, and in the steps behind it: the logits of the model over each text."""
    m = _model(name, "int4")
    rng = torch.Generator().manual_seed(7)
    text = lambda k: torch.randint(0, m.shape["vocab"], (k,), generator=rng, dtype=torch.int32).to(DEV)
    a = Answers(m, n_seq=6, n_blocks=60, block=16, max_blocks=12, width=4, e4m3=e4m3)
    prompt = text(75)
    a.add(prompt, _i32([75, 0, 0, 0, 0, 0]))
    a.fork(_i32([0, 0, 0, 0, -1, -1]))
    texts = [prompt] * 4 + [prompt[:0]] * 2
    nothing = torch.zeros(0, dtype=torch.int32, device=DEV)

    def step(added, where):
        new = [text(k) if k > 0 else nothing for k in added]
        for i, x in enumerate(new):
            texts[i] = torch.cat([texts[i], x]) if added[i] >= 0 else nothing
        got = a.add(torch.cat(new), _i32(added)).clone()
        assert int(a.state[2]) == 0 and a.lengths.tolist() == [t.numel() for t in texts]
        for i in where:
            want = _logits(m, texts[i])
            assert _far(got[i], want[-1]) <= max(0.1 if e4m3 else 2e-2, 2 * _apart(m, texts[i], want)), i
        _check_cache(a)

    step([1, 2, 1, 1, 0, 0], [0, 1, 2, 3])
    step([-1, 0, 0, 0, 0, 0], [])
    assert a.shared.tolist()[0] == 64
    step([length, 1, 3, 1, 9, 0], [0, 1, 2, 3, 4])
    step([1, 1, 1, 1, 1, 2], [0, 1, 2, 3, 4, 5])
    step([0, 0, -1, 0, 0, 0], [])
    step([1, 1, length, 1, 1, 1], [0, 1, 2, 3, 4, 5])


# ------------------------------------------------------------------ what an Answers keeps, without a device ----
def _on_the_host(monkeypatch, events):
    """Answers over host tensors, its calls of the library only noted: (name, scratch)."""
    note = lambda name: lambda *a, **k: events.append((name, k.get("scratch")))
    for name in ("qzo_cache_fork", "qzo_cache_copy", "qzo_cache_compact", "qzo_cache_plan", "qzo_answer"):
        monkeypatch.setattr(qb, name, note(name))
    monkeypatch.setattr(qb, "make_cache", lambda *a: None)
    monkeypatch.setattr(qb, "qzo_answer_workspace_bytes", lambda *a: 256)
    monkeypatch.setattr(torch.cuda, "synchronize", note("synchronize"))
    model = types.SimpleNamespace(shape=dict(d_model=128, n_heads=2, vocab=8, n_layers=1), scales=torch.zeros(1), handle=None)
    return lambda **k: Answers(model, **dict(dict(n_seq=8, n_blocks=2100, block=16), **k))


@pytest.mark.parametrize("width", [None, 4])
def test_scratch_of_forks_is_there_before_any_call(monkeypatch, width):
    """A call that makes it may be captured: nothing has zeroed it then before the graph's first replay."""
    events = []
    a = _on_the_host(monkeypatch, events)(width=width)
    for turn in range(2):
        room = a._fork_room
        assert room.numel() >= qb.qzo_cache_fork_scratch_bytes(8, a.free.numel(), 2100) and not room.any() and a.copies.shape[0] >= max(8, a.free.numel() // 2)
        events.clear()
        a.fork(torch.arange(8, dtype=torch.int32))
        a.add(torch.zeros(3, dtype=torch.int32), torch.tensor([3] + [0] * 7, dtype=torch.int32))
        a.compact()
        assert all(s is room for name, s in events if name in ("qzo_cache_fork", "qzo_cache_compact")) and len(events) >= 5
        a.state[0] = a.free.numel()
        a.resize(3000)


@gpu
@pytest.mark.parametrize("first", ["add", "fork", "resize"])
def test_a_captured_first_fork_before_eager_ones(first):
    """A step is captured, the prompts are read by eager calls, then it is replayed: beyond the fork's small form, in memory that was not zero."""
    m = _model("tiny", "int4")
    text = torch.randint(0, 1024, (200,), generator=torch.Generator().manual_seed(8), dtype=torch.int32).to(DEV)
    runs = []
    for captured in (False, True):
        torch.cuda.empty_cache()
        filled = [torch.full((1 << n,), -1, dtype=torch.int32, device=DEV) for n in range(7, 24)]
        del filled
        a = Answers(m, n_seq=8, n_blocks=2100 if first != "resize" else 50, block=16, width=4 if first != "fork" else None)
        if first == "resize":
            a.resize(17000)                     # the table's columns stay: the small form's pool is what it is beyond
        one, tokens, parents = _i32([1] * 4 + [0] * 4), text[:4].contiguous(), _i32([0, 1, 2, 3, -1, -1, -1, -1])

        def step():
            if first == "fork":
                a.fork(parents)
            a.add(tokens, one)

        a.rows(200)
        torch.cuda.synchronize()
        if captured:
            g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            with torch.cuda.graph(g, stream=side):
                step()
        a.add(text[:90].contiguous(), _i32([30, 20, 25, 15, 0, 0, 0, 0]))
        a.fork(_i32([0, 0, 2, 2, 1, -1, -1, -1]))
        found = []
        for _ in range(4):
            g.replay() if captured else step()
            torch.cuda.synchronize()
            assert int(a.state[2]) == 0
            _check_cache(a)
            found += [a.logits.clone(), a.lengths.clone(), a.tables.clone()]
            a.add(text[:5].contiguous(), _i32([2, 1, 1, 1, 0, 0, 0, 0]))
            found.append(a.logits.clone())
        runs.append(found)
    assert all(torch.equal(x, y) for x, y in zip(*runs))


def test_a_resize_waits_before_it_begins(monkeypatch):
    """Steps may be under way on any stream: the device is waited for before the pool is made compact, and behind whatever resize does."""
    events = []
    a = _on_the_host(monkeypatch, events)(width=4)
    for n_blocks, held in ((3000, 5), (100, 100), (2, 3)):
        a.state[0] = a.free.numel() - held
        events.clear()
        if n_blocks < held:
            with pytest.raises(ValueError):
                a.resize(n_blocks)
        else:
            a.resize(n_blocks)
        names = [name for name, _ in events]
        assert names[:2] == ["synchronize", "qzo_cache_compact"] and names[-1] == "synchronize"


@gpu
def test_a_resize_behind_steps_on_another_stream():
    m = _model("tiny", "int4")
    text = torch.randint(0, 1024, (400,), generator=torch.Generator().manual_seed(9), dtype=torch.int32).to(DEV)
    runs, side, kept = [], torch.cuda.Stream(), []       # kept: what the side stream reads stays until it has been read

    def counts(x):
        kept.append(_i32(x))
        return kept[-1]

    for stream in (None, side):
        a = Answers(m, n_seq=4, n_blocks=60, block=16, max_blocks=12, width=2)
        torch.cuda.synchronize()
        found = []
        for n_blocks in (40, 80, 50):
            for added in ([60, 0, 40, 0], [1, 0, 1, 0], [3, 0, 2, 0]):
                a.add(text[:sum(added)].contiguous(), counts(added), stream)
            a.fork(counts([0, 0, 2, 2]), stream)
            a.resize(n_blocks)
            _check_cache(a)
            a.add(text[:8].contiguous(), counts([1, 3, 2, 2]), stream)
            torch.cuda.synchronize()
            found.append(a.logits.cpu())
            a.add(text[:0], counts([-1] * 4), stream)
        runs.append(found)
    assert all(torch.equal(x, y) for x, y in zip(*runs))


# ------------------------------------------------------------------ sums of rows that rise ----
def _rising_rows(n, vocab, seed):
    """Rows of tiles that lie higher than the ones before, by 2 to 120, anywhere from -3000 to 3000: few or many logits near the highest."""
    rng = np.random.default_rng(seed)
    off, rise = rng.choice([-3000, -400, -376, -100, -24.25, 0, 100, 400, 776, 3000], n), rng.choice([2, 5, 5.6, 8, 20, 40, 41, 41.5, 42, 44, 50, 60], n)
    x = off[:, None] + rng.standard_normal((n, vocab)) * 0.1
    x[:, 1024:2048] += rise[:, None]
    for i in range(n):
        k = (1, 17, 1000)[i % 3]
        x[i, 2048:2048 + k] += rise[i] + rng.uniform(0, 6)
        x[i, 3000] += rise[i] + rng.uniform(0, 8)
        if i % 5 == 0:
            x[i, 3500] += 2 * rise[i]
    x[0] = -np.inf                              # 776, many at 816, the highest 820: the reference moves by 44 while the sum is all of the others'
    x[0, :1024], x[0, 1024:2024], x[0, 2048] = 776, 816, 820
    return torch.tensor(x, dtype=torch.float32, device=DEV).to(torch.bfloat16)


@gpu
@pytest.mark.parametrize("n,vocab", [(1200, 4096), (1100, 8200), (20, 4096)])
def test_select_sums_up_rows_that_rise(n, vocab):
    """One beam a prompt, whose score tells its row's sum; more than 1024 rows: a row is one wavefront's, whose reference moves."""
    logits = _rising_rows(n, vocab, n)
    _check_select(logits, 1, [0.0] * n, [0] * n, [0] * n, np.zeros((n, 0), np.int32), -1, 0.0)


@gpu
@pytest.mark.parametrize("n,vocab", [(1100, 4096), (12, 40000), (1100, 9)])
def test_select_of_large_logits(n, vocab):
    """From 2^13 to the largest number, of either sign, at the beginning, late, everywhere, and as masks."""
    rng = np.random.default_rng(n + vocab)
    x = rng.standard_normal((n, vocab))
    for i in range(n):
        v = 2.0 ** rng.uniform(13, 127.9)
        at = [0, vocab - 1, vocab // 2, rng.integers(0, vocab)][i % 4]
        kind = i % 6
        if kind == 0:
            x[i, at] = v
        elif kind == 1:
            x[i, at:at + 3] = [v, v, v * 0.75][:len(x[i, at:at + 3])]
        elif kind == 2:
            x[i] = -v * (1 + rng.random(vocab))
        elif kind == 3:
            x[i, rng.random(vocab) < 0.5] = -v            # a mask
        elif kind == 4:
            x[i, :-1] = -3.3895e38                        # all but one
        else:
            x[i] *= v / 8
    x = np.clip(x, -3.3895e38, 3.3895e38)
    _check_select(torch.tensor(x, dtype=torch.float32, device=DEV).to(torch.bfloat16), 1, [0.0] * n, [0] * n, [0] * n, np.zeros((n, 0), np.int32), -1, 0.0)


# ------------------------------------------------------------------ steps that cannot be made ----
@gpu
@pytest.mark.parametrize("width", [None, 2])
def test_a_refused_step_ends_nobody(width):
    """Sequences that share blocks are ended by a fork ahead of the plan: a plan that is refused takes that back, and a refused fork refuses the step."""
    m = _model("tiny", "int4")
    text = torch.randint(0, 1024, (400,), generator=torch.Generator().manual_seed(10), dtype=torch.int32).to(DEV)
    runs = []
    for refused in (False, True):
        a = Answers(m, n_seq=5, n_blocks=14, block=16, max_blocks=10, width=width)
        a.add(text[:70].contiguous(), _i32([40, 0, 30, 0, 0]))
        a.fork(_i32([0, 0, 2, 2, 2]))
        a.add(text[:5].contiguous(), _i32([1] * 5))
        found = []
        for turn in range(3):
            if refused:
                kept = lambda: [x.clone() for x in (a.lengths, a.free[:int(a.state[0])], a.tables, a.state[:1])] + ([] if width is None else [a.shared.clone()])
                before = kept()
                for added, rows, status in [([-1, 1, 200, 0, 0], 201, qb.QZO_ERR_SHAPE), ([0, 0, 118, -1, 1], 119, qb.QZO_ERR_WORKSPACE), ([-1, 0, 9, -2, 1], 9, qb.QZO_ERR_SHAPE),
                                            ([-1, 0, 0, -1, 1], 0, qb.QZO_ERR_SHAPE)]:
                    out = a.add(text[:rows].contiguous(), _i32(added))
                    assert a.state.tolist()[1:] == [0, status, 0] and (out == 0).all()
                    assert all(torch.equal(x, y) for x, y in zip(before, kept()))
                n_free = int(a.state[0])
                a.state[0] = 14                      # more than there can be, so that nothing can be given back
                before[1], before[3] = a.free[:14].clone(), a.state[:1].clone()
                a.add(text[:2].contiguous(), _i32([-1, -1, -1, 1, 1]))
                assert a.state.tolist() == [14, 0, qb.QZO_ERR_ARG, 0] and all(torch.equal(x, y) for x, y in zip(before, kept()))
                a.state[0] = n_free
            found.append(a.add(text[:6].contiguous(), _i32([1, -1 if turn == 1 else 1, 1, 3 if turn == 1 else 2, 1 if turn < 2 else -1])).clone())
            assert int(a.state[2]) == 0
            found.append(a.lengths.clone())
            _check_cache(a)
        runs.append(found)
    assert all(torch.equal(x, y) for x, y in zip(*runs))


@gpu
def test_captured_steps_of_which_some_are_refused():
    """The step is the same graph, whatever it is given: replayed with counts that fit and that do not, eager work in between."""
    m = _model("tiny", "int4")
    text = torch.randint(0, 1024, (400,), generator=torch.Generator().manual_seed(11), dtype=torch.int32).to(DEV)
    counts = [[1, 1, 1, 1], [-1, 1, 1, 5], [1, 2, -1, 1], [-1, -1, 4, 0], [0, 4, 0, 0], [-1, 1, 2, 1]]
    runs = []
    for captured in (False, True):
        a = Answers(m, n_seq=4, n_blocks=12, block=16, max_blocks=6, width=4)
        tokens, added = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
        a.add(text[:60].contiguous(), _i32([60, 0, 0, 0]))
        a.fork(_i32([0] * 4))
        torch.cuda.synchronize()
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                a.add(tokens, added)
        found = []
        for i in range(12):
            added.copy_(_i32(counts[i % 6]))
            tokens.copy_(text[4 * i:4 * i + 4])
            g.replay() if captured else a.add(tokens, added)
            torch.cuda.synchronize()
            m.forward_loss(text.view(1, -1)[:, :40].contiguous(), 1, 1e-3, 1)
            found += [a.logits.clone(), a.lengths.clone(), a.state.clone(), a.shared.clone(), a.tables.clone()]
            _check_cache(a)
        assert {int(x[2]) for x in found[2::5]} >= {0, qb.QZO_ERR_SHAPE}
        runs.append(found)
    assert all(torch.equal(x, y) for x, y in zip(*runs))


# ------------------------------------------------------------------ how many groups there may be ----
def test_more_groups_than_attend_together_are_refused(monkeypatch):
    """When the pools are made, not in a step that has planned already.  Groups of one attend by themselves."""
    make = _on_the_host(monkeypatch, [])
    for n, width in ((4097, 2), (8192, 3), (2049 * 3, 3)):
        with pytest.raises(ValueError):
            make(n_seq=n, n_blocks=4, width=width)
    for n, width in ((4096, 2), (2048 * 3, 3), (8192, 4)):
        assert make(n_seq=n, n_blocks=4, width=width).shared.numel() == -(-n // width) <= qb.MAX_GROUPS
    seen = []
    monkeypatch.setattr(qb, "qzo_answer", lambda *a, group_starts, shared: seen.append((group_starts, shared)))
    for width in (1, 2):
        a = make(n_seq=4096, n_blocks=4, width=width)
        a.add(torch.zeros(3, dtype=torch.int32), torch.zeros(4096, dtype=torch.int32))
        assert (a.group_starts.numel(), a.shared.numel()) == (4096 // width + 1, 4096 // width)
    assert seen[0] == (None, None) and seen[1] == (a.group_starts, a.shared)


@gpu
def test_beams_of_more_prompts_than_groups():
    """2100 prompts with one beam each: greedy continuations, every step's tokens those of the highest logits."""
    m, n = _model("tiny", "int4"), 2100
    b = Beams(m, n, 1, n_blocks=2 * n, max_new=4, block=16, max_blocks=2)
    tokens = torch.randint(0, m.shape["vocab"], (3 * n,), generator=torch.Generator().manual_seed(12), dtype=torch.int32).to(DEV)
    b.start(tokens, _i32([3] * n))
    for i in range(3):
        logits = b.answers.logits.float()
        assert torch.equal(logits.gather(1, b.tokens.long()[:, None])[:, 0], logits.max(1).values) and int(b.failed) == 0
        b.step()
    _check_cache(b.answers)
    with pytest.raises(ValueError):
        Beams(m, n, 2, n_blocks=n, max_new=4, block=16, max_blocks=2)
