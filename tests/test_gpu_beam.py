"""The beam selection on the GPU against float64."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import operators as O
from paper_2507_01021_amd import binding

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, binding.DTYPE_F32), "bf16": (torch.bfloat16, binding.DTYPE_BF16)}


def run(b, dtype, logits, scores, width, n, stride=0):
    groups = scores.numel() // width
    out = [torch.full((groups + 1, n), 7, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    b.run(logits.data_ptr(), DT[dtype][1], groups, width, n, scores.data_ptr(), *(x.data_ptr() for x in out), stride)
    torch.cuda.synchronize()
    assert all((x[groups] == 7).all() for x in out)
    return [x[:groups] for x in out]


def check(got, logits, scores, width, n, suppress=()):
    l, c = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    for g in range(len(c) // width):
        rows = slice(g * width, (g + 1) * width)
        p, t, s = O.continuations(c[rows], l[rows], n, suppress)
        assert np.array_equal(got[0][g].cpu().numpy(), p), g
        assert np.array_equal(got[1][g].cpu().numpy(), t), g
        # exponentials 2e-12 each, rounded once
        x = got[2][g].double().cpu().numpy()
        ok = np.isfinite(s)
        assert np.array_equal(np.isfinite(x), ok)
        assert (np.abs(x[ok] - s[ok]) <= 2.0 ** -24 * np.abs(s[ok]) + 1e-11).all()


def make(dtype, rows, V, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    logits = (torch.randn(rows, V, generator=g, device="cuda") * 2.5).to(DT[dtype][0])
    return logits, torch.rand(rows, generator=g, device="cuda") * -20


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 33, 515, 4099, 51865])
@pytest.mark.parametrize("groups,width,n", [(1, 1, 1), (1, 5, 10), (3, 2, 4), (2, 8, 16), (1, 32, 64), (2, 1, 64)])
def test_against_float64(dtype, V, groups, width, n):
    logits, scores = make(dtype, groups * width, V, V + n)
    suppress = [0, V // 2] if V > 4 else []
    b = binding.Beam(V, groups * width)
    b.options(suppress)
    check(run(b, dtype, logits, scores, width, n), logits, scores, width, n, suppress)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beams_that_are_not_there(dtype):
    V, width, n = 5003, 5, 10
    logits, scores = make(dtype, 6 * width, V, 1)
    scores[1:5] = -math.inf  # a first step
    scores[5:10] = -math.inf  # no beam at all
    scores[12], scores[14] = math.nan, math.inf
    logits[1:5] = math.nan  # not read
    logits[20] = -math.inf  # a beam without a continuation
    logits[25:30, 3:] = -math.inf  # fewer than n
    logits[15:20, ::7] = math.nan
    b = binding.Beam(V, 30)
    got = run(b, dtype, logits, scores, width, n)
    check(got, logits, scores, width, n)
    assert (got[0][1] == -1).all() and (got[1][1] == -1).all() and (got[2][1] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [9, 700, 20001])
def test_equal_logits_go_by_beam_and_id(dtype, V):
    """Rows of one value, rows and beams that are alike, zeros of both signs."""
    width, n = 4, 20
    logits = torch.full((5 * width, V), 1.25, device="cuda").to(DT[dtype][0])
    scores = torch.full((5 * width,), -3.0, device="cuda")
    scores[width: 2 * width] = torch.tensor([-4.0, -3.0, -5.0, -3.0])
    logits[2 * width: 3 * width] = torch.randint(0, 3, (V,), device="cuda").to(logits.dtype)  # alike, with ties
    logits[3 * width: 4 * width] = torch.where(torch.arange(V, device="cuda") % 2 == 0, -0.0, 0.0).to(logits.dtype)
    logits[4 * width:] = torch.randn(V, device="cuda").to(logits.dtype)
    b = binding.Beam(V, 5 * width)
    check(run(b, dtype, logits, scores, width, n), logits, scores, width, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["up", "down", "steps"])
def test_sorted_logits(dtype, order):
    """Every id larger than all before it, and the other way round."""
    V, width, n = 30011, 3, 7
    x = torch.arange(V, device="cuda").double() / V * 600 - 300
    if order == "down":
        x = x.flip(0)
    if order == "steps":  # plateaus
        x = (x / 40).floor() * 40
    logits = torch.stack([x, x + 1, x * 0.5]).to(DT[dtype][0])
    scores = torch.tensor([-1.0, -2.0, -2.5], device="cuda")
    b = binding.Beam(V, 3)
    check(run(b, dtype, logits, scores, width, n), logits, scores, width, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_and_extreme_logits(dtype):
    V, width, n = 3001, 3, 8
    logits, scores = make(dtype, 5 * width, V, 3)
    logits[0, [5, 2000, 77]] = math.inf
    logits[4, 2999] = math.inf
    low, high = torch.finfo(logits.dtype).min, torch.finfo(logits.dtype).max
    logits[6], logits[7, 9], logits[8] = low, high, -1e4
    logits[9], logits[10, ::2], logits[11] = high, low, torch.linspace(-1e30, 1e30, V, device="cuda").to(logits.dtype)
    logits[12], logits[13, 4], logits[14] = 500.0, 1000.0, logits[14] * 100
    b = binding.Beam(V, 15)
    check(run(b, dtype, logits, scores, width, n), logits, scores, width, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 5), (0, 1), (7, 64)])
def test_rows_at_any_address(dtype, offset, pad):
    V, width, groups, n = 1021, 3, 4, 6
    t = DT[dtype][0]
    flat = torch.full((offset + groups * width * (V + pad),), 1e4, device="cuda").to(t)
    view = flat[offset:].view(groups * width, V + pad)
    logits, scores = make(dtype, groups * width, V, offset)
    view[:, :V] = logits
    b = binding.Beam(V, groups * width)
    check(run(b, dtype, view, scores, width, n, V + pad), logits, scores, width, n)


def test_many_groups():
    """More rows than one launch takes; a group's choice is the same in any call."""
    V, width, n, groups = 997, 5, 10, 230
    logits, scores = make("f32", groups * width, V, 9)
    b = binding.Beam(V, groups * width)
    got = run(b, "f32", logits, scores, width, n)
    check(got, logits, scores, width, n)
    for g in (0, 101, 102, 229):
        one = run(b, "f32", logits[g * width:], scores[g * width: (g + 1) * width], width, n)
        assert all(torch.equal(x[0], y[g]) for x, y in zip(one, got))
    again = run(b, "f32", logits, scores, width, n)
    assert all(torch.equal(x, y) for x, y in zip(again, got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_rows_of_equal_logits(dtype):
    """More equal logits than any list holds, in every piece of a row and over all of
    them; runs of equal ones among others."""
    V, width, n = 200003, 4, 64
    logits, scores = make(dtype, 4 * width, V, 11)
    logits[:width] = -2.0
    scores[:width] = -3.0
    logits[width: 2 * width] = torch.tensor([0.0, 1.0, 1.0, 0.0], device="cuda")[:, None]
    scores[width: 2 * width] = torch.tensor([-1.0, -1.0, -7.0, -1.0])
    logits[2 * width: 3 * width, 150000:199000] = 30.0  # all in some pieces
    logits[3 * width, ::3], logits[3 * width + 1, 1::5] = 9.0, 30.0
    b = binding.Beam(V, 4 * width)
    check(run(b, dtype, logits, scores, width, n), logits, scores, width, n)
    b.options([0, 1, V - 1, 150000])
    check(run(b, dtype, logits, scores, width, n), logits, scores, width, n, [0, 1, V - 1, 150000])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_widest_call(dtype):
    """32 beams of 2^20 ids; then more groups than one launch takes of such rows."""
    V = 1 << 20
    logits, scores = make(dtype, 32, V, 12)
    b = binding.Beam(V, 70)
    check(run(b, dtype, logits, scores, 32, 64), logits, scores, 32, 64)
    logits = torch.cat([logits, logits.flip(0), logits[:6] + 1]).contiguous()
    scores = torch.rand(70, device="cuda") * -20
    got = run(b, dtype, logits, scores, 2, 5)
    for g in (0, 15, 16, 31, 32, 34):
        rows = slice(2 * g, 2 * g + 2)
        check([x[g: g + 1] for x in got], logits[rows], scores[rows], 2, 5)


def test_two_handles_at_once():
    """Graphs of two handles, replayed on two streams beside each other."""
    made = []
    for V, width, n, dtype in ((50001, 5, 10, "bf16"), (20000, 8, 16, "f32")):
        b = binding.Beam(V, 3 * width)
        logits, scores = make(dtype, 3 * width, V, V)
        out = [torch.zeros(3, n, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
        st = torch.cuda.Stream()
        torch.cuda.synchronize()
        b.set_stream(st.cuda_stream)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            b.run(logits.data_ptr(), DT[dtype][1], 3, width, n, scores.data_ptr(), *(x.data_ptr() for x in out))
        made.append((b, logits, scores, out, st, g, width, n, dtype, V))
    for i in range(4):
        for b, logits, scores, out, st, g, width, n, dtype, V in made:
            new, sc = make(dtype, 3 * width, V, i)
            logits.copy_(new)
            scores.copy_(sc)
        torch.cuda.synchronize()
        for _ in range(3):
            for b, logits, scores, out, st, g, width, n, dtype, V in made:
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        for b, logits, scores, out, st, g, width, n, dtype, V in made:
            check(out, logits, scores, width, n)


def test_close_scores():
    """Continuations of different beams that differ by a few 2^-40 of a score: far
    less than fp32 tells apart."""
    V, n = 2048, 6
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    logits = torch.randn(3, V, generator=g, device="cuda") - 8
    logits[:, 100] = 4.0
    for eps in (2.0 ** -22, 2.0 ** -21):  # the sums differ by such a share of one of 2048 ids
        logits[1] = logits[0]
        logits[2] = logits[0]
        i = int(logits[0, 200:].argmax()) + 200
        logits[1, i] *= 1 + eps
        logits[2, i] *= 1 - eps
        scores = torch.full((3,), -1.0, device="cuda")
        b = binding.Beam(V, 3)
        check(run(b, "f32", logits, scores, 3, n), logits, scores, 3, n)


def test_recorded_runs_and_streams():
    """A replay takes the logits, scores and suppressed ids of its time."""
    V, width, groups, n = 5000, 5, 3, 10
    b = binding.Beam(V, 64)
    logits, scores = make("bf16", groups * width, V, 4)
    out = [torch.zeros(groups, n, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    b.set_stream(st.cuda_stream)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        b.run(logits.data_ptr(), binding.DTYPE_BF16, groups, width, n, scores.data_ptr(), *(x.data_ptr() for x in out))
        for f in (lambda: b.options([1]), lambda: b.set_stream(None)):
            with pytest.raises(binding.WhisperError) as e:
                f()
            assert e.value.status == binding.E_STATE
    suppress = []
    for i in range(4):
        if i:
            new, sc = make("bf16", groups * width, V, 40 + i)
            logits.copy_(new)
            scores.copy_(sc)
        if i >= 2:
            suppress = [int(out[1][0, 0]), 17, V - 1][: i]
            b.options(suppress)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        check(out, logits, scores, width, n, suppress)
        (torch.randn(64, 64, device="cuda") @ torch.randn(64, 64, device="cuda")).sum().item()
    b.set_stream(None)
    check(run(b, "bf16", logits, scores, width, n), logits, scores, width, n, suppress)


@pytest.mark.parametrize("bits", [0, 4, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_beam_search(dtype, bits):
    """Selection, reordered sequences, appends and attention together: a small decoder's
    beams of two utterances over several steps. What every beam's sequence
    holds is the keys and values of its own tokens, and each choice is that of
    its logits."""
    t, code = DT[dtype]
    V, width, groups, D, H = 300, 4, 2, 64, 2
    n_seq = groups * width
    g = torch.Generator(device="cuda")
    g.manual_seed(bits)
    embed, out_w = torch.randn(V, H * D, generator=g, device="cuda"), torch.randn(H * D, V, generator=g, device="cuda")
    wq, wk, wv = (torch.randn(H * D, H * D, generator=g, device="cuda") * (H * D) ** -0.5 for _ in range(3))
    cache = binding.Cache(code, 1, H, H, D, 32, 40, n_seq, 200, 400, bits=bits)
    beam = binding.Beam(V, n_seq)
    beam.options([0])

    def kv(tokens):
        x = embed[torch.tensor(tokens, device="cuda")]
        return (x @ wq).to(t).contiguous(), (x @ wk).to(t).contiguous(), (x @ wv).to(t).contiguous()

    prompts = [[5, 9, 200] * 11, [7] * 30]  # 33 tokens, 30 tokens
    history = [None] * n_seq
    heads = [u * width for u in range(groups)]
    cache.extend(heads, [len(p) for p in prompts])
    q, k, v = kv(sum(prompts, []))
    out = torch.empty_like(q)
    cache.append(0, k.data_ptr(), v.data_ptr())
    cache.attend(0, q.data_ptr(), out.data_ptr())
    last = [sum(len(p) for p in prompts[: u + 1]) - 1 for u in range(groups)]
    scores = torch.full((n_seq,), -math.inf, device="cuda")
    logits = torch.zeros(n_seq, V, device="cuda")
    for u in range(groups):
        scores[u * width] = 0
        logits[u * width] = out[last[u]].float() @ out_w * 0.2
        history[u * width] = prompts[u]
    for step in range(10):
        parents, tokens, new = run(beam, "f32", logits, scores, width, 2 * width)
        check((parents, tokens, new), logits, scores, width, 2 * width, [0])
        src, toks, keep = [], [], []
        for u in range(groups):
            rows = [(int(parents[u, i]), int(tokens[u, i]), float(new[u, i])) for i in range(2 * width)]
            rows = [r for r in rows if r[1] != 1][: width]  # id 1 ends an utterance
            src += [u * width + r[0] for r in rows]
            toks += [r[1] for r in rows]
            keep += [r[2] for r in rows]
        cache.reorder(list(range(n_seq)), src)
        history = [history[s] + [x] for s, x in zip(src, toks)]
        cache.extend(list(range(n_seq)), [1] * n_seq)
        q, k, v = kv(toks)
        out = torch.empty_like(q)
        cache.append(0, k.data_ptr(), v.data_ptr())
        cache.attend(0, q.data_ptr(), out.data_ptr())
        logits = out.float() @ out_w * 0.2
        scores = torch.tensor(keep, device="cuda")
        torch.cuda.synchronize()
    lens = [len(h) for h in history]
    kb, vb = (torch.empty(sum(lens), H * D, dtype=t, device="cuda") for _ in range(2))
    cache.read(0, list(range(n_seq)), kb.data_ptr(), vb.data_ptr())
    torch.cuda.synchronize()
    at = 0
    for s, h in enumerate(history):
        # (a product of one row may round differently from that of many: rows as they were appended)
        q1, k1, v1 = kv(h)
        for got, x in ((kb, k1), (vb, v1)):
            y = got[at: at + len(h)].double().cpu().numpy().reshape(-1, H, D)
            x = x.double().cpu().numpy().reshape(-1, H, D)
            step = O.packed(x, bits)[1].repeat(64, -1) if bits else np.abs(x) * torch.finfo(t).eps
            # half a step, half of one if x falls on the other side of a rounding (of the step itself: as much again)
            assert (np.abs(y - x) <= step * 1.5 + np.abs(x) * torch.finfo(t).eps + 1e-5).all(), s
        at += len(h)
    assert len({tuple(h) for h in history}) == n_seq  # beams differ
