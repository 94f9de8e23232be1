"""Device-memory plumbing around the C ABI: uploads a tensor table, owns the
scale arena and the workspace, and forwards to the binding.  No arithmetic of
the method happens here."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as qb
from . import synth


class DeviceModel:
    """A model bound to device tensors.  `tensors` follow qzo_model_create's
    order: bf16 tensors for the fixed parts, uint8 [N, K/2] for packed int4."""

    def __init__(self, shape: dict, tensors, scale_arena: torch.Tensor):
        self.shape = dict(shape)
        self.tensors = tensors
        self.scales = scale_arena
        self.handle = qb.qzo_model_create(shape, tensors, scale_arena)
        self._ws = None
        self._ws_key = None
        self.result = torch.zeros(8, dtype=torch.int32, device=scale_arena.device)
        self.loss = torch.zeros(2, dtype=torch.float32, device=scale_arena.device)
        self.dense_master = None

    @classmethod
    def from_host(cls, shape: dict, host_tensors, host_scales, device="cuda:0"):
        """host_tensors: numpy fp32 arrays holding bf16-exact values, or uint8
        packed weights; host_scales: fp32 array of bf16-exact scales."""
        dev = []
        for a in host_tensors:
            t = torch.from_numpy(np.ascontiguousarray(a))
            dev.append(t.to(device) if t.dtype in (torch.uint8, torch.int32) else t.to(device).to(torch.bfloat16))
        arena = torch.from_numpy(np.ascontiguousarray(host_scales, dtype=np.float32)).to(device).to(
            torch.float16 if shape.get("scale_fp16") else torch.bfloat16)
        return cls(shape, dev, arena)

    @classmethod
    def from_host_codebook(cls, shape: dict, table, device="cuda:0"):
        """Codebook variant.  table: (name, kind, array) with kind 'bf16' (fp32 holding bf16
        values), 'codes' (uint16 [N,K/8]), 'codebook' (fp32 holding fp16 values, [65536,8]) or
        'chscale' (fp32 holding fp16 values, [N]); channel scales form the fp16 arena."""
        dev, scales = [], []
        for _, kind, a in table:
            a = np.ascontiguousarray(a)
            if kind == "chscale":
                scales.append(a.reshape(-1))
            elif kind == "codes":
                dev.append(torch.from_numpy(a.view(np.int16)).to(device))
            elif kind == "codebook":
                dev.append(torch.from_numpy(a).to(device).to(torch.float16))
            else:
                dev.append(torch.from_numpy(a).to(device).to(torch.bfloat16))
        arena = torch.from_numpy(np.concatenate(scales).astype(np.float32)).to(device).to(torch.float16)
        return cls(dict(shape, quant=1), dev, arena)

    @classmethod
    def synthetic(cls, shape: dict, seed: int, device="cuda:0", asym=False, nf4=False):
        """Random-init model built on the device: weights ~ N(0, 0.02) drawn by
        torch, quantized by the library's RTN kernel (Eq. 3), tensor by tensor.
        asym: the zero-point variant (quant = 2) as the 4-bit checkpoints of Sec. 4.1 hold it: the
        library's asymmetric RTN kernel gives every group a zero-point and an fp16 scale (each
        output row's weights are shifted by up to 0.03 so that the zero-points spread)."""
        if asym:
            shape = dict(shape, quant=2, scale_fp16=1)
        if nf4:
            # NormalFloat-4: uniform random level indices, block-64 scales ~ U(0.03, 0.09) (the absmax
            # of 64 weights ~ N(0, 0.02)): the shapes, sizes and work of such a checkpoint
            shape = dict(shape, quant=3, group=64)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        d, V = shape["d_model"], shape["vocab"]
        llama = shape["arch"] == "llama"
        n_scales = qb.qzo_model_scale_count(shape)
        arena = torch.empty(n_scales, dtype=torch.float16 if asym else torch.bfloat16, device=device)
        off = 0

        def fixed(*sz, mean=0.0, std=0.02):
            return (torch.randn(*sz, generator=gen, device=device) * std + mean).to(torch.bfloat16)

        def quant(N, K):
            nonlocal off
            if nf4:
                n = N * (K // 64)
                arena[off:off + n] = (torch.rand(n, generator=gen, device=device) * 0.06 + 0.03).to(torch.bfloat16)
                off += n
                return [torch.randint(0, 256, (N, K // 2), generator=gen, device=device, dtype=torch.uint8)]
            w = torch.randn(N, K, generator=gen, device=device) * 0.02
            q = torch.empty(N, K // 2, dtype=torch.uint8, device=device)
            n = N * (K // 128)
            if asym:
                w += 0.03 * torch.sin(torch.arange(N, device=device, dtype=torch.float32))[:, None]
                zp = torch.empty(N, K // 128, dtype=torch.uint8, device=device)
                qb.qzo_rtn_quantize_asym(w, q, zp, arena[off:off + n].view(N, K // 128))
                off += n
                return [q, zp]
            qb.qzo_rtn_quantize(w, q, arena[off:off + n].view(N, K // 128))
            off += n
            return [q]

        tensors = [fixed(V, d)]
        if not llama:
            tensors.append(fixed(shape["max_seq"], d))
        lin = synth.quantized_linears(shape)
        for _ in range(shape["n_layers"]):
            if llama:
                tensors += ([fixed(d, mean=1.0, std=0.1)] + quant(*lin[0][1:]) + quant(*lin[1][1:]) +
                            [fixed(d, mean=1.0, std=0.1)] + quant(*lin[2][1:]) + quant(*lin[3][1:]))
            else:
                tensors += ([fixed(d, mean=1.0, std=0.1), fixed(d)] + quant(*lin[0][1:]) +
                            [fixed(lin[0][1])] + quant(*lin[1][1:]) + [fixed(d)] +
                            [fixed(d, mean=1.0, std=0.1), fixed(d)] + quant(*lin[2][1:]) +
                            [fixed(lin[2][1])] + quant(*lin[3][1:]) + [fixed(d)])
        tensors.append(fixed(d, mean=1.0, std=0.1))
        if not llama:
            tensors.append(fixed(d))
        tensors.append(fixed(V, d))
        torch.cuda.synchronize()
        assert off == n_scales
        return cls(shape, tensors, arena)

    @classmethod
    def synthetic_codebook(cls, shape: dict, seed: int, device="cuda:0"):
        """Random-init codebook-variant model built on the device: uniform 16-bit codes,
        one fp16 [65536, 8] codebook ~ N(0, 0.02) per linear, fp16 channel scales ~ U(0.5, 1.5)."""
        assert shape["arch"] == "llama"
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        d, V = shape["d_model"], shape["vocab"]
        cfg = dict(shape, quant=1)
        arena = (torch.rand(qb.qzo_model_scale_count(cfg), generator=gen, device=device) + 0.5).to(torch.float16)

        def fixed(*sz, mean=0.0, std=0.02):
            return (torch.randn(*sz, generator=gen, device=device) * std + mean).to(torch.bfloat16)

        def lin(N, K):
            codes = torch.randint(-32768, 32768, (N, K // 8), generator=gen, device=device, dtype=torch.int16)
            cb = (torch.randn(65536, 8, generator=gen, device=device) * 0.02).to(torch.float16)
            return [codes, cb]

        tensors = [fixed(V, d)]
        ql = synth.quantized_linears(shape)
        for _ in range(shape["n_layers"]):
            tensors += [fixed(d, mean=1.0, std=0.1)] + lin(*ql[0][1:]) + lin(*ql[1][1:])
            tensors += [fixed(d, mean=1.0, std=0.1)] + lin(*ql[2][1:]) + lin(*ql[3][1:])
        tensors += [fixed(d, mean=1.0, std=0.1), fixed(V, d)]
        torch.cuda.synchronize()
        return cls(cfg, tensors, arena)

    def workspace(self, batch, seq):
        if self._ws_key != (batch, seq):
            n = qb.qzo_workspace_bytes(self.handle, batch, seq)
            self._ws = torch.empty(n, dtype=torch.uint8, device=self.scales.device)
            self._ws_key = (batch, seq)
        return self._ws

    def forward_loss(self, tokens, seed, eps, sign, stream=None) -> torch.Tensor:
        ws = self.workspace(*tokens.shape)
        out = self.loss[0:1] if sign > 0 else self.loss[1:2]
        qb.qzo_forward_loss(self.handle, tokens, seed, eps, sign, ws, out, stream)
        return out

    def step(self, tokens, seed, eps, eta, clip, stream=None) -> torch.Tensor:
        ws = self.workspace(*tokens.shape)
        qb.qzo_step(self.handle, tokens, seed, eps, eta, clip, ws, self.result, stream)
        return self.result

    def enable_joint(self):
        """Joint mode: an fp32 master of every 16-bit tensor (table order), copied from the tensors;
        from here on the library rewrites those tensors from the master."""
        parts = [t.reshape(-1) for t in self.tensors if t.dtype in (torch.bfloat16, torch.float16)]
        self.dense_master = torch.cat(parts).to(torch.float32)       # a copy: dtype conversion only
        assert self.dense_master.numel() == qb.qzo_model_dense_count(self.shape)
        self.joint_table = torch.empty(qb.qzo_model_joint_table_bytes(self.shape), dtype=torch.uint8,
                                       device=self.scales.device)
        qb.qzo_model_enable_joint(self.handle, self.dense_master, self.joint_table)
        self._ws = None                                              # the workspace layout may differ
        self._ws_key = None
        return self.dense_master

    def step_joint(self, tokens, seed, eps, eta, eta_dense, clip, stream=None) -> torch.Tensor:
        ws = self.workspace(*tokens.shape)
        qb.qzo_step_joint(self.handle, tokens, seed, eps, eta, eta_dense, clip, ws, self.result, stream)
        return self.result

    def set_int4_path(self, mode: int):
        """0: by token count, 1: always the fused kernel, 2: always expand-then-multiply."""
        qb.qzo_model_set_int4_path(self.handle, mode)
        self._ws = None                                              # the workspace layout depends on it
        self._ws_key = None

    def apply_update(self, seed, eta, d_clipped, stream=None):
        qb.qzo_model_apply_update(self.handle, seed, eta, d_clipped, stream)

    def close(self):
        if self.handle is not None:
            qb.qzo_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Answers:
    """Sequences that a DeviceModel continues: the pools of all layers, block tables, the free list, the lengths.  One call of `add`
    per step; everything stays on the device.  width: sequences i * width .. (i + 1) * width - 1 are a group that may come to share what
    they begin with (`fork`), and attend to that together; the last group may be smaller.  At most 2048 groups, but any number of one sequence each,
    which attend by themselves."""

    def __init__(self, model: DeviceModel, n_seq: int, n_blocks: int, block: int = 32, max_blocks: int | None = None, e4m3: bool = False,
                 k_scale=None, v_scale=None, width: int | None = None):
        if width is not None and width > 1 and -(-n_seq // width) > qb.MAX_GROUPS:
            raise ValueError(f"groups of {width} of {n_seq} sequences are more than {qb.MAX_GROUPS}")
        sh, dev = model.shape, model.scales.device
        dh = sh["d_model"] // sh["n_heads"]
        self.model, self.block, self.vocab = model, block, sh["vocab"]
        size = (sh["n_layers"], n_blocks, sh["n_heads"], block, dh)
        self.k, self.v = (torch.empty(size, dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16, device=dev) for _ in range(2))
        self.scales = (k_scale, v_scale)
        self.cache = qb.make_cache(self.k[0], self.v[0], *self.scales)
        i32 = dict(dtype=torch.int32, device=dev)
        self.tables = torch.full((n_seq, max_blocks or n_blocks), -1, **i32)
        self.free = torch.arange(n_blocks, **i32)
        n_groups = 0 if width is None else -(-n_seq // width)
        # what a step that is refused leaves as it was, in one tensor: the state, lengths, what the groups share
        at = 4 + (n_seq + 3) // 4 * 4
        self._kept_whole = torch.zeros(at + n_groups, **i32)
        self.state, self.lengths = self._kept_whole[:4], self._kept_whole[4:4 + n_seq]
        self.state[0] = n_blocks
        self.starts = torch.zeros(n_seq + 1, **i32)
        self.logits = torch.zeros(n_seq, self.vocab, dtype=torch.bfloat16, device=dev)
        self._kept = [(torch.zeros(0, **i32), torch.zeros(0, **i32), torch.zeros(0, dtype=torch.uint8, device=dev))]
        self.group_starts = self.shared = None
        if width is not None:
            self.group_starts = torch.arange(n_groups + 1, **i32).mul_(width).clamp_(max=n_seq)
            self.shared = self._kept_whole[at:]
        self.forked, self.together = width is not None, width is not None and width > 1
        self._own = torch.arange(n_seq, **i32)
        self._make_fork_room()

    def rows(self, n_tokens: int, stream=None):
        """Slots, positions and workspace of steps of that many rows, from buffers that double as they are outgrown; the earlier ones
        are kept for the graphs that were captured with them.  New ones are made on the stream that uses them."""
        slots, positions, ws = self._kept[-1]
        need = qb.qzo_answer_workspace_bytes(self.model.handle, n_tokens, len(self.lengths), self.together)
        if slots.numel() < n_tokens or ws.numel() < need:
            dev, n = self.free.device, max(n_tokens, 2 * slots.numel())
            with torch.cuda.stream(stream):
                slots, positions = (torch.zeros(n, dtype=torch.int32, device=dev) for _ in range(2))
                ws = torch.empty(max(need, 2 * ws.numel()), dtype=torch.uint8, device=dev)
            self._kept.append((slots, positions, ws))
        return slots[:n_tokens], positions[:n_tokens], ws

    def add(self, tokens: torch.Tensor, added: torch.Tensor, stream=None) -> torch.Tensor:
        """tokens int32 [rows], the new tokens sequence by sequence, padded at the end; added int32 [n_seq], how many each adds (negative:
        it ends and gives its blocks back).  A step without tokens ends sequences and runs no model.  Returns the logits bf16 [n_seq, vocab]
        of the last new tokens: `logits`, the same buffer every step, which the next one overwrites (a graph that holds the step writes it, too;
        keep a copy of what is to outlive a step).  Whether the step could be planned is in state[2], where the caller may look (not QZO_OK: nothing has
        changed, no sequence has ended, the logits are zeros)."""
        if not self.forked:
            return self._add(tokens, added, stream)
        with torch.cuda.stream(stream):         # what ends may share its blocks: they are given back by a fork
            before = self._kept_whole.clone()
            parents = torch.where(added < 0, -1, self._own)
        self.fork(parents, stream)
        with torch.cuda.stream(stream):         # none is negative; but where the fork was refused those that were still are, and the plan is refused as well
            added = torch.maximum(added, self.state[2:3])
        self._add(tokens, added, stream)
        with torch.cuda.stream(stream):         # a plan that is refused takes the fork back: no more of the free list's valid part than its end was written
            before[1:4] = self.state[1:4]
            torch.where(self.state[2:3] == 0, self._kept_whole, before, out=self._kept_whole)
        return self.logits

    def _add(self, tokens, added, stream=None):
        slots, positions, ws = self.rows(max(1, tokens.numel()), stream)
        if tokens.numel() == 0:                 # a plan has room for one token: a sequence that would add any adds more, so that it is refused
            with torch.cuda.stream(stream):
                added = torch.where(added > 0, 2, added)
                self.logits.zero_()
        qb.qzo_cache_plan(self.lengths, added, self.block, self.tables, self.free, self.state, self.lengths, self.starts, slots, positions,
                          self.state, stream)
        if tokens.numel():
            qb.qzo_answer(self.model.handle, tokens, self.cache, self.tables, self.lengths, self.starts, slots, positions, ws, self.logits, stream,
                          group_starts=self.group_starts if self.together else None, shared=self.shared if self.together else None)
        return self.logits

    def _make_fork_room(self):
        """List of copies and scratch of forks and compactions, made with the pools: were it made in the first call, and that one captured, the
        scratch would be zero from the graph's first replay on only, and eager calls may come before it."""
        n, n_blocks, dev = len(self.lengths), self.free.numel(), self.free.device
        self.copies = torch.zeros(max(n, n_blocks // 2), 4, dtype=torch.int32, device=dev)
        self._fork_room = torch.zeros(qb.qzo_cache_fork_scratch_bytes(n, n_blocks, self.tables.shape[1]), dtype=torch.uint8, device=dev)

    def fork(self, parents: torch.Tensor, stream=None):
        """parents int32 [n_seq]: sequence i goes on from what sequence parents[i] is (negative: it ends).  Full blocks are shared, open ones copied.
        An `add` that was captured before the first fork does not know that blocks may be shared (with a width it does).
        Whether there were blocks for that is in state[2], as for `add` (not QZO_OK: nothing has changed)."""
        self.forked = True
        qb.qzo_cache_fork(parents, self.block, self.lengths, self.tables, self.free, self.state, self.copies, group_starts=self.group_starts,
                          shared=self.shared, scratch=self._fork_room, stream=stream)
        qb.qzo_cache_copy(self.cache, self.copies[:len(self.lengths)], layers=self.k.shape[0], count=self.state, stream=stream)

    def compact(self, stream=None):
        """The blocks in use to the front of the pools: those from n_blocks - state[0] on are free."""
        qb.qzo_cache_compact(self.block, self.lengths, self.tables, self.free, self.tables, self.state, self.copies, scratch=self._fork_room, stream=stream)
        qb.qzo_cache_copy(self.cache, self.copies, layers=self.k.shape[0], count=self.state, stream=stream)

    def resize(self, n_blocks: int):
        """Pools of another number of blocks: memory given back to a training step between answers, or more of it.  Waits for the device, before (steps
        may be under way on any stream) and behind what it does; what was captured with the old pools is no longer valid.  ValueError: the
        sequences hold more blocks than that (nothing has changed but their places).  Where memory runs out for the new pools, the old ones are gone."""
        torch.cuda.synchronize(self.free.device)
        self.compact()
        free, had = int(self.state[0]), self.free.numel()
        used = had - free
        if n_blocks < max(1, used):
            torch.cuda.synchronize(self.free.device)
            raise ValueError(f"{used} blocks are in use")
        for name in ("k", "v"):                 # one pool after the other: the old one's memory is free before the next is made
            old = getattr(self, name)
            new = torch.empty((old.shape[0], n_blocks, *old.shape[2:]), dtype=old.dtype, device=old.device)
            new.view(torch.uint8)[:, :used].copy_(old.view(torch.uint8)[:, :used])
            setattr(self, name, new)
            self.cache = None
            del old
        self.cache = qb.make_cache(self.k[0], self.v[0], *self.scales)
        i32 = dict(dtype=torch.int32, device=self.free.device)
        self.free = torch.full((n_blocks,), -1, **i32)
        self.free[:n_blocks - used] = torch.arange(n_blocks - 1, used - 1, -1, **i32)
        self.state[0] = n_blocks - used
        self._make_fork_room()
        torch.cuda.synchronize(self.free.device)


class Beams:
    """Beam search with a DeviceModel: `width` beams for each of n_prompts prompts, over a cache whose blocks they share.  `search` runs it;
    `start` and `step` are its parts, and a step, which leaves everything on the device, can be captured into a graph."""

    def __init__(self, model: DeviceModel, n_prompts: int, width: int, n_blocks: int, max_new: int, end_token: int = -1, length_penalty: float = 0.0,
                 block: int = 32, max_blocks: int | None = None, e4m3: bool = False, k_scale=None, v_scale=None):
        n, dev = n_prompts * width, model.scales.device
        i32 = dict(dtype=torch.int32, device=dev)
        self.answers = Answers(model, n, n_blocks, block, max_blocks, e4m3, k_scale, v_scale, width)
        self.width, self.end_token, self.length_penalty = width, end_token, length_penalty
        self.scores, self.history = torch.full((n,), -float("inf"), device=dev), torch.full((n, max_new), -1, **i32)
        self.counts, self.ended, self.parents, self.chosen, self.tokens, self.added = (torch.zeros(n, **i32) for _ in range(6))
        self.room = torch.zeros(qb.qzo_beam_select_scratch_bytes(n_prompts, width, self.answers.vocab), dtype=torch.uint8, device=dev)
        self.failed = torch.zeros(1, **i32)

    def _go_on(self, logits, stream):
        a = self.answers
        with torch.cuda.stream(stream):
            torch.minimum(self.failed, a.state[2:3], out=self.failed)
        qb.qzo_beam_select(logits, self.width, self.scores, self.counts, self.ended, self.history, self.parents, self.chosen, self.tokens, self.added,
                           end_token=self.end_token, length_penalty=self.length_penalty, scratch=self.room, stream=stream)
        a.fork(self.parents, stream)
        with torch.cuda.stream(stream):
            torch.minimum(self.failed, a.state[2:3], out=self.failed)

    def start(self, tokens: torch.Tensor, lengths: torch.Tensor, stream=None):
        """tokens int32, the prompts one behind the other; lengths int32 [n_prompts], at least 1.  The beams of before are given up."""
        a = self.answers
        with torch.cuda.stream(stream):
            nobody = torch.full_like(self.parents, -1)
            added = torch.zeros_like(self.added)
            added[::self.width] = lengths
            self.scores.fill_(-float("inf"))
            self.scores[::self.width] = 0.0
            for t in (self.counts, self.ended, self.failed):
                t.zero_()
            self.history.fill_(-1)
        a.fork(nobody, stream)
        self._go_on(a._add(tokens, added, stream), stream)

    def step(self, stream=None):
        """Every beam that has not ended by a token, and the next beams."""
        self._go_on(self.answers._add(self.tokens, self.added, stream), stream)

    def search(self, tokens: torch.Tensor, lengths: torch.Tensor, look_every: int = 8):
        """Up to max_new tokens behind every prompt; now and then looks whether all beams have ended.  Returns history [n_prompts, width, max_new] (tokens,
        behind a beam's last one -1), counts and scores [n_prompts, width], the best beam first.  RuntimeError: the cache has too few blocks."""
        self.start(tokens, lengths)
        for i in range(1, self.history.shape[1]):
            if i % look_every == 0 and bool(self.ended.all()):
                break
            self.step()
        if int(self.failed):
            raise RuntimeError(f"the sequences did not fit the cache (status {int(self.failed)})")
        column = torch.arange(self.history.shape[1], device=self.history.device)
        history = torch.where(column < self.counts[:, None], self.history, -1)
        return history.view(-1, self.width, self.history.shape[1]), self.counts.view(-1, self.width), self.scores.view(-1, self.width)
