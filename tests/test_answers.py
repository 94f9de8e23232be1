"""Sequences continued by a model out of a paged cache, against the model's own forward over the whole sequences.

Both round activations to bf16 at the same places, some twelve times a layer, each a relative error of at most 2^-8 and some
2^-9 / sqrt(3) as a standard deviation, which add up like independent ones: sqrt(12 layers) * 1.1e-3, 0.6e-2 of a
logit vector's norm at two layers for the difference of two such paths; 2e-2 is the bar that losses are held to as well.  An
e4m3 cache rounds keys and values by up to 2^-4 (standard deviation 2^-5 / sqrt(3), 1.8e-2) more."""
import ctypes as C
import dataclasses

import pytest
import torch

from paper_2505_13430_amd import binding as qb
from paper_2505_13430_amd import synth
from paper_2505_13430_amd.model import Answers, DeviceModel

DEV = "cuda:0"
gpu = pytest.mark.gpu
WIDE_HEADS = dict(arch="llama", n_layers=2, d_model=256, n_heads=2, d_ffn=512, vocab=520, max_seq=160)


def _shape(name):
    return dict(WIDE_HEADS) if name == "wide_heads" else dict(synth.SHAPES[name], max_seq=160)


def _model(name, fmt, seed=3):
    shape = _shape(name)
    if fmt == "codebook":
        return DeviceModel.synthetic_codebook(shape, seed, DEV)
    m = DeviceModel.synthetic(shape, seed, DEV, asym=fmt == "zp", nf4=fmt == "nf4")
    if fmt == "expanded":
        m.set_int4_path(2)
    return m


def _logits(m, tokens):
    """Logits behind every position of one sequence, by the forward that trains."""
    d, S = m.shape["d_model"], tokens.numel()
    hidden = torch.zeros(S, d, dtype=torch.bfloat16, device=DEV)
    qb.qzo_debug_forward(m.handle, tokens.view(1, S), 0, 0.0, 1, m.workspace(1, S), m.loss, hidden)
    return hidden.float() @ m.tensors[-1].float().T.contiguous()


def _apart(m, tokens, want):
    """How far two forwards over the same sequence with the same weights, bit for bit, are apart where they add up in another order: the
    largest distance of a row's logits between an int4 model's fused linears and its expanded ones.  Where activations nearly
    cancel that is far more than the roundings themselves (tiny, zero-points: 0.14 for one of these sequences).  Two right
    results are each at most about that far from the exact one, so twice that from one another (triangle inequality)."""
    m.set_int4_path(2)
    other = _logits(m, tokens)
    m.set_int4_path(0)
    return float(((other - want).norm(dim=1) / want.norm(dim=1)).max())


def _far(got, want):
    return float((got.float() - want).norm() / want.norm())


@gpu
@pytest.mark.parametrize("name,fmt,e4m3", [
    ("tiny", "int4", False), ("tiny", "int4", True), ("wide_heads", "int4", False), ("wide_heads", "int4", True), ("tiny_opt", "int4", False),
    ("tiny_opt", "int4", True), ("tiny", "zp", False), ("tiny", "nf4", False), ("wide_heads", "codebook", False), ("wide_heads", "codebook", True),
    ("wide_heads", "expanded", False), ("tiny_opt", "zp", False)])
def test_continued_sequences_follow_the_forward(name, fmt, e4m3):
    """Prompts of different lengths at once (more than 64 tokens in all), a long one later, single tokens, one sequence that ends and
    whose place another takes; rows of padding."""
    m = _model(name, fmt)
    rng = torch.Generator().manual_seed(4)
    texts = [torch.randint(0, m.shape["vocab"], (n,), generator=rng, dtype=torch.int32).to(DEV) for n in (90, 30, 47, 120)]
    want = [_logits(m, t) for t in texts]
    a = Answers(m, n_seq=3, n_blocks=30, block=16, max_blocks=10, e4m3=e4m3)
    seats, done = [0, 1, 2], [0, 0, 0]            # which text sits where, how much of it is in
    bars = [0.1 if e4m3 else 2e-2] * 4
    if fmt in ("int4", "zp"):
        bars = [max(b, 2 * _apart(m, t, w)) for b, t, w in zip(bars, texts, want)]
    steps = [([60, 1, 13], 80), ([1, 1, 1], 3), ([1, 20, 1], 22), ([1, -1, 1], 4), ([1, 75, 1], 77), ([1, 1, 1], 3), ([0, 1, 0], 1), ([1, 40, 1], 64)] + [([1, 1, 1], 3)] * 3
    for added, rows in steps:
        tokens = torch.zeros(rows, dtype=torch.int32, device=DEV)
        at = 0
        for i, n in enumerate(added):
            if n < 0:
                seats[i], done[i] = 3, 0
                continue
            tokens[at:at + n] = texts[seats[i]][done[i]:done[i] + n]
            at, done[i] = at + n, done[i] + n
        got = a.add(tokens, torch.tensor(added, dtype=torch.int32, device=DEV))
        assert a.state.tolist()[1:3] == [at, 0] and a.lengths.tolist() == done
        for i, n in enumerate(added):
            if n > 0:
                assert _far(got[i], want[seats[i]][done[i] - 1]) <= bars[seats[i]], (added, i)
            else:
                assert not bool(got[i].any())


@gpu
@pytest.mark.parametrize("name,fmt,seed", [("tiny", "int4", 3), ("wide_heads", "int4", 3), ("tiny_opt", "int4", 3), ("tiny_opt", "zp", 3), ("tiny", "zp", 4)])
def test_continued_sequences_within_a_fixed_bar(name, fmt, seed):
    """Two sequences of well-conditioned models, in parts and token by token: within 2e-2, whatever two right forwards differ by; here they
    differ by no more than half of that (no sequence's activations nearly cancel), which is looked at, too."""
    m = _model(name, fmt, seed)
    rng = torch.Generator().manual_seed(4)
    texts = [torch.randint(0, m.shape["vocab"], (n,), generator=rng, dtype=torch.int32).to(DEV) for n in (90, 30)]
    want = [_logits(m, t) for t in texts]
    assert max(_apart(m, t, w) for t, w in zip(texts, want)) <= 1e-2
    a, done = Answers(m, n_seq=2, n_blocks=10, block=16), [0, 0]
    for added in [(70, 3), (1, 25), (17, 0)] + [(1, 1)] * 2:
        parts = [t[d:d + n] for t, d, n in zip(texts, done, added)]
        got = a.add(torch.cat(parts), torch.tensor(added, dtype=torch.int32, device=DEV))
        done = [d + n for d, n in zip(done, added)]
        for i in range(2):
            if added[i]:
                assert _far(got[i], want[i][done[i] - 1]) <= 2e-2, (added, i)
    assert a.lengths.tolist() == [90, 30]


@gpu
def test_answers_use_the_scales_as_they_are():
    """After an update of the scales the answers are those of the updated model."""
    m = _model("tiny", "int4")
    text = torch.arange(40, dtype=torch.int32, device=DEV)
    before = _logits(m, text)
    m.apply_update(5, 1e-3, 1.0)                                  # steps of 1e-3 |z| at scales of some 8e-3
    after = _logits(m, text)
    a = Answers(m, n_seq=1, n_blocks=4, block=16)
    got = a.add(text, torch.tensor([40], dtype=torch.int32, device=DEV))
    assert _far(got[0], after[-1]) <= 2e-2 < _far(got[0], before[-1])


@gpu
def test_answers_of_a_jointly_trained_model():
    """A perturbed forward in joint mode leaves the 16-bit tensors perturbed; an answer is the unperturbed model's."""
    m = _model("tiny", "int4")
    m.enable_joint()
    text = torch.arange(40, dtype=torch.int32, device=DEV)
    want = _logits(m, text)
    m.forward_loss(text.view(1, -1), 3, 0.05, 1)
    a = Answers(m, n_seq=1, n_blocks=4, block=16)
    assert _far(a.add(text, torch.tensor([40], dtype=torch.int32, device=DEV))[0], want[-1]) <= 2e-2


@gpu
def test_a_step_that_cannot_be_planned_changes_nothing():
    m = _model("wide_heads", "int4")
    a = Answers(m, n_seq=2, n_blocks=3, block=16)
    ones = torch.ones(40, dtype=torch.int32, device=DEV)
    a.add(ones[:20], torch.tensor([17, 3], dtype=torch.int32, device=DEV))
    k = a.k.clone()
    got = a.add(ones, torch.tensor([16, 24], dtype=torch.int32, device=DEV))
    assert a.state.tolist() == [0, 0, qb.QZO_ERR_WORKSPACE, 0] and a.lengths.tolist() == [17, 3] and not bool(got.any())
    assert torch.equal(a.k.view(torch.int16), k.view(torch.int16))
    got = a.add(ones[:2], torch.tensor([1, 1], dtype=torch.int32, device=DEV))      # and it goes on
    assert a.state.tolist()[2] == 0 and _far(got[0], _logits(m, ones[:18])[-1]) <= 2e-2


@gpu
def test_profile_of_an_answer():
    """Launches and work by class: the attention's work, which depends on lengths that only the device knows, is 0, its launches are
    one a layer; rotations count as class 4, beside the embedding."""
    m = _model("tiny", "int4")
    sh = m.shape
    a = Answers(m, n_seq=2, n_blocks=8, block=16)
    added = torch.tensor([30, 5], dtype=torch.int32, device=DEV)
    a.rows(35)
    qb.qzo_profile_begin(100)
    a.add(torch.arange(35, dtype=torch.int32, device=DEV), added)
    got = {k: qb.qzo_profile_collect(v) for k, v in qb.PROFILE_KINDS.items()}
    assert (got["attention"]["launches"], got["attention"]["work"]) == (sh["n_layers"], 0.0) and got["attention"]["total_ms"] > 0
    assert (got["embed"]["launches"], got["embed"]["work"]) == (1 + sh["n_layers"], 0.0)
    assert (got["lmhead_ce"]["launches"], got["lmhead_ce"]["work"]) == (1, 2.0 * 2 * sh["vocab"] * sh["d_model"])
    assert got["w4a16_gemm"]["work"] == 2.0 * 35 * sh["n_layers"] * (4 * sh["d_model"] ** 2 + 3 * sh["d_model"] * sh["d_ffn"])


@gpu
def test_logits_are_one_buffer():
    """What `add` returns is `logits`, also after a longer step; a copy is what outlives the next step."""
    m = _model("tiny", "int4")
    a = Answers(m, n_seq=1, n_blocks=4, block=16)
    text = torch.arange(50, dtype=torch.int32, device=DEV)
    got = a.add(text[:1], torch.tensor([1], dtype=torch.int32, device=DEV))
    first = got.clone()
    again = a.add(text[1:].clone(), torch.tensor([49], dtype=torch.int32, device=DEV))
    assert again.data_ptr() == got.data_ptr() == a.logits.data_ptr() and torch.equal(got, again) and not torch.equal(got, first)


@gpu
def test_a_step_that_only_ends_sequences():
    """No token at all: the blocks go back, the logits are zeros, what goes on goes on; tokens that are not there are refused."""
    m = _model("tiny", "int4")
    a, none = Answers(m, n_seq=2, n_blocks=4, block=16), torch.zeros(0, dtype=torch.int32, device=DEV)
    text = torch.arange(40, dtype=torch.int32, device=DEV)

    def step(tokens, *added):
        return a.add(tokens, torch.tensor(added, dtype=torch.int32, device=DEV))

    step(text[:35], 30, 5)
    got = step(none, -1, 0)
    assert a.state.tolist() == [3, 0, 0, 0] and a.lengths.tolist() == [0, 5] and not bool(got.any())
    for added in ((0, 1), (1, -1), (0, 2 ** 31 - 1)):
        step(none, *added)
        assert a.state.tolist() == [3, 0, qb.QZO_ERR_SHAPE, 0] and a.lengths.tolist() == [0, 5]
    got = step(torch.cat([text, text[35:36]]), 40, 1)
    assert a.state.tolist() == [0, 41, 0, 3] and a.lengths.tolist() == [40, 6]
    assert _far(got[0], _logits(m, text)[-1]) <= 2e-2
    step(none, -1, -1)
    assert a.state.tolist() == [4, 0, 0, 0] and sorted(a.free.tolist()) == [0, 1, 2, 3]


@gpu
@pytest.mark.parametrize("name", ["tiny", "tiny_opt"])
def test_captured_steps_answer_as_eager_ones(name):
    """A step of one token a sequence captured into a graph, the next token chosen inside it: replays, with the program's own eager work
    in between, write the same text bit for bit."""
    m = _model(name, "int4")
    prompt = torch.arange(24, dtype=torch.int32, device=DEV) * 7
    counts = torch.tensor([10, 14], dtype=torch.int32, device=DEV)
    one = torch.ones(2, dtype=torch.int32, device=DEV)
    texts = []
    for captured in (False, True):
        a = Answers(m, n_seq=2, n_blocks=20, block=16)
        a.rows(2)
        tokens = a.add(prompt, counts).argmax(1).to(torch.int32)
        text = [tokens.clone()]

        def step():
            tokens.copy_(a.add(tokens, one).argmax(1))

        torch.cuda.synchronize()
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
        for i in range(30):
            g.replay() if captured else step()
            torch.cuda.synchronize()
            m.forward_loss(prompt.view(1, -1), 1, 1e-3, 1)         # eager work of the same model
            text.append(tokens.clone())
        texts.append(torch.stack(text))
        assert a.lengths.tolist() == [40, 44] and a.state.tolist()[2] == 0
    assert torch.equal(texts[0], texts[1])


# ------------------------------------------------------------------ refusals, on the host ----
@dataclasses.dataclass
class _Unbacked:
    """A tensor of a model table that host-only calls can be handed: an aligned address nothing reads."""
    n: int
    e: int
    is_cuda = True

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return self.n

    def element_size(self):
        return self.e


@gpu
def test_buffers_are_made_on_the_stream_that_uses_them():
    """A step on a stream of its own while the current one is held up: what the buffers are cleared with must not come after the plan."""
    m = _model("tiny", "int4")
    text = torch.randint(0, m.shape["vocab"], (40,), generator=torch.Generator().manual_seed(9), dtype=torch.int32).to(DEV)
    added = torch.tensor([40], dtype=torch.int32, device=DEV)
    want = Answers(m, n_seq=1, n_blocks=4).add(text, added).clone()
    a, side = Answers(m, n_seq=1, n_blocks=4), torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.randn(4096, 4096, device=DEV)
    for _ in range(20):
        busy = busy @ busy.T.contiguous() * 1e-4
    got = a.add(text, added, stream=side)
    side.synchronize()
    assert torch.equal(got.cpu(), want.cpu()) and torch.equal(a._kept[-1][1][:40].cpu(), torch.arange(40, dtype=torch.int32))
    torch.cuda.synchronize()
    assert torch.equal(a._kept[-1][1][:40].cpu(), torch.arange(40, dtype=torch.int32))


@gpu
def test_workspace_elsewhere_is_refused():
    """Host memory, and memory with gaps, as the workspace of an answer."""
    m = _model("tiny", "int4")
    a, tokens = Answers(m, n_seq=1, n_blocks=4, block=16), torch.zeros(2, dtype=torch.int32, device=DEV)
    slots, positions, ws = a.rows(2)
    for bad in (torch.zeros(ws.numel(), dtype=torch.uint8), torch.zeros(2 * ws.numel(), dtype=torch.uint8, device=DEV)[::2]):
        with pytest.raises(AssertionError):
            qb.qzo_answer(m.handle, tokens, a.cache, a.tables, a.lengths, a.starts, slots, positions, bad, a.logits)


def _host_model(vocab=1024):
    shape = dict(synth.SHAPES["tiny"], n_layers=1, vocab=vocab)
    d, F = shape["d_model"], shape["d_ffn"]
    sizes = [(vocab * d, 2), (d, 2), (3 * d * d // 2, 1), (d * d // 2, 1), (d, 2), (F * d, 1), (d * F // 2, 1), (d, 2), (vocab * d, 2)]
    return qb.qzo_model_create(shape, [_Unbacked(*s) for s in sizes], _Unbacked(qb.qzo_model_scale_count(shape), 2))


@pytest.mark.parametrize("over,status", [
    (dict(model=None), qb.QZO_ERR_ARG), (dict(tokens=None), qb.QZO_ERR_ARG), (dict(cache=None), qb.QZO_ERR_ARG), (dict(starts=None), qb.QZO_ERR_ARG),
    (dict(slots=24), qb.QZO_ERR_ALIGN), (dict(workspace=16), qb.QZO_ERR_ALIGN), (dict(n_tokens=0), qb.QZO_ERR_SHAPE), (dict(n_seq=0), qb.QZO_ERR_SHAPE),
    (dict(n_seq=8193), qb.QZO_ERR_SHAPE), (dict(n_tokens=1 << 22), qb.QZO_ERR_SHAPE), (dict(max_blocks=0), qb.QZO_ERR_SHAPE),
    (dict(bytes=1024), qb.QZO_ERR_WORKSPACE), (dict(cache=dict(kv_heads=2)), qb.QZO_ERR_SHAPE), (dict(cache=dict(head_dim=128)), qb.QZO_ERR_SHAPE),
    (dict(cache=dict(block=24)), qb.QZO_ERR_SHAPE), (dict(cache=dict(type=3)), qb.QZO_ERR_UNSUPPORTED)])
def test_answer_refuses(over, status):
    model = _host_model()
    v = dict(model=model, tokens=16, n_tokens=4, n_seq=2, cache={}, tables=16, max_blocks=4, lengths=16, starts=16, slots=16, positions=16,
             workspace=256, bytes=1 << 40, logits=16)
    v.update(over)
    if v["cache"] is not None:
        c = dict(struct_size=C.sizeof(qb.qzo_cache), type=0, n_blocks=8, block=16, kv_heads=4, head_dim=64, k_dev=16, v_dev=16, k_scale_dev=None,
                 v_scale_dev=None)
        c.update(v["cache"])
        cache = qb.qzo_cache(*c.values())
        v["cache"] = C.addressof(cache)
    assert qb.lib().qzo_answer(*v.values(), None) == status and qb.lib().qzo_last_error()
    qb.qzo_model_destroy(model)


def test_answer_workspace():
    model = _host_model()
    few, more = qb.qzo_answer_workspace_bytes(model, 1, 1), qb.qzo_answer_workspace_bytes(model, 300, 8)
    assert few % 256 == 0 and more > few
    odd = _host_model(vocab=1023 * 4 + 2)
    with pytest.raises(qb.QzoError) as e:
        qb.qzo_answer_workspace_bytes(odd, 1, 1)
    assert e.value.status == qb.QZO_ERR_SHAPE
    for m in (model, odd):
        qb.qzo_model_destroy(m)
