"""Several sampled candidates of one segment: paged self-attention caches,
forked slots and drawn tokens, together and one by one.

A row's result depends on its own slot alone, so a fork's logits are, bit for
bit, those of a slot that was encoded by itself and fed the same tokens; paged
contexts are checked against the oracle with the tolerances of the others."""
import numpy as np
import pytest

from paper_2507_01021_amd import binding, synth

from parity import TOL, bands, check_free_run, check_tokens, oracle_run, rel_row_err
from test_gpu_sampler import choose

pytestmark = pytest.mark.gpu

PROMPT_LENS = [1, 4, 70, 130]


def model(name, **kw):
    shape = {"tiny": synth.TINY, "base": synth.BASE}[name].with_(**kw)
    W = synth.make_weights(shape, 0)
    return shape, W, synth.pack_blob(W)


def segments(shape, n_new, seed, lens=PROMPT_LENS):
    segs = synth.fixed_batch(shape, [16000 + 40000 * i for i in range(len(lens))], n_new, seed=seed)
    base = synth.prompt_for(shape)
    for s, n in zip(segs, lens):
        s.prompt = (base + [400 + 37 * k % 9000 for k in range(n)])[:n]
    return segs


def forced_logits(ctx, slots, segs, tokens, prefilled):
    """Logits of the generated positions of each slot, fed tokens[k]."""
    out = []
    for k, (slot, s) in enumerate(zip(slots, segs)):
        if not prefilled:
            for _ in range(len(s.prompt) - 1):
                assert ctx.decode_step([slot])[0] == -1
        out.append(np.stack([ctx.decode_step([slot], forced=[int(t)], logits=True)[1][0] for t in tokens[k]]))
    return out


@pytest.mark.parametrize("prefill", [0, 1])
def test_paged_context_against_oracle(prefill):
    shape, W, blob = model("tiny")
    segs = segments(shape, 6, 31)
    ref = oracle_run(W, shape, segs, n_new=6)
    with binding.Context(blob, max_slots=4, prefill=prefill, paged=1) as ctx:
        ctx.encode(segs, [2, 0, 3, 1])
        lgs = forced_logits(ctx, [2, 0, 3, 1], segs, [r["tokens"] for r in ref], prefill)
        got = ctx.transcribe(segs)
    for lg, r, g in zip(lgs, ref, got):
        assert rel_row_err(lg, r["logits"]).max() < TOL["f32"]
        check_tokens(np.argmax(lg, axis=-1), r["logits"], gpu_logits=lg, min_strict=3)
        check_free_run(g["tokens"], r["tokens"], r["logits"], bands(r["logits"], lg), min_agree=3)


def test_paged_bf16_against_fixed_caches():
    """Logits of both kinds of cache agree within the bf16 tolerance; whether
    the prompt is fed step by step or prefilled changes no bit."""
    shape, W, blob = model("base", n_enc=2)
    segs = segments(shape, 8, 32)
    toks = [[500 + 11 * j + k for j in range(8)] for k in range(4)]
    out = {}
    for paged, prefill in ((0, 0), (1, 0), (1, 1)):
        with binding.Context(blob, max_slots=4, paged=paged, prefill=prefill) as ctx:
            ctx.encode(segs, [0, 1, 2, 3])
            out[paged, prefill] = forced_logits(ctx, [0, 1, 2, 3], segs, toks, prefill)
    for a, b, c in zip(out[0, 0], out[1, 0], out[1, 1]):
        assert rel_row_err(b, a).max() < TOL["bf16"]
        assert np.array_equal(b, c)


def test_paged_two_chains_and_refills():
    """40 slots in two chains, more segments than slots, prompts of one to nine
    tokens: the same tokens as each segment's by itself."""
    shape, W, blob = model("base", n_enc=1, n_dec=2)
    segs = synth.uniform_batch(shape, 60, 5, seed=24)
    base = synth.prompt_for(shape)
    for k, s in enumerate(segs):
        n = 1 + k % 9
        s.prompt = (base + [300 + 13 * j for j in range(n)])[:n]
        s.max_new_tokens = 4 + k % 90
    outs = []
    for prefill in (0, 1):
        with binding.Context(blob, max_slots=40, paged=1, prefill=prefill, refill_min=4, max_encode_batch=1) as ctx:
            outs.append([r["tokens"] for r in ctx.transcribe(segs)])
            again = [ctx.transcribe([segs[k]])[0]["tokens"] for k in (0, 41, 59)]
    for a, b in zip(*outs):
        assert np.array_equal(a, b)
    for k, t in zip((0, 41, 59), again):
        assert np.array_equal(outs[1][k], t)


@pytest.mark.parametrize("name", ["tiny", "base"])
@pytest.mark.parametrize("prefill", [0, 1])
@pytest.mark.parametrize("before", [0, 1, 5])
def test_forks_equal_slots_encoded_by_themselves(name, prefill, before):
    """Forked right after the encode, after a step and after five, with a prompt
    that ends inside a page and at a page's end."""
    shape, W, blob = model(name, n_enc=1)
    for n_prompt in (3, 64, 65 - before):
        seg = segments(shape, 9, 33, [n_prompt])[0]
        first = n_prompt - 1 if not prefill else 0  # steps that feed the prompt
        toks = [[700 + 13 * j * (k + 1) for j in range(9)] for k in range(3)]
        for k in (1, 2):
            toks[k][: max(0, before - first)] = toks[0][: max(0, before - first)]
        with binding.Context(blob, max_slots=5, prefill=prefill, paged=1) as ctx:
            for k in range(3):
                ctx.encode([seg], [k])
            want = forced_logits(ctx, [0, 1, 2], [seg] * 3, toks, prefill)
            ctx.encode([seg], [3])
            lg = [[], [], []]
            for i in range(before):
                t, l = ctx.decode_step([3], forced=[toks[0][max(0, i - first)]], logits=True)
                if i >= first:
                    for x in lg:
                        x.append(l[0])
            ctx.fork(3, [0, 4])  # slots 0..2 are idle again; 3 goes on as candidate 0
            slots, order = [3, 0, 4], [0, 1, 2]
            for i in range(before, first + 9):
                g = i - first
                t, l = ctx.decode_step(slots, forced=[toks[k][max(0, g)] for k in order], logits=True)
                for k in order:
                    if g >= 0:
                        lg[k].append(l[k])
            for k in order:
                assert np.array_equal(np.stack(lg[k]), want[k]), (n_prompt, k)
                assert ctx.slot_tokens(slots[k]).size == 9


def test_fork_outlives_its_source():
    """The source ends and its slot is encoded anew while forks go on; a fork
    is forked again; cross-attention caches stay with who reads them."""
    shape, W, blob = model("tiny", n_enc=1, n_dec=2)
    a, b = segments(shape, 12, 34, [4, 4])
    toks = [600 + 7 * j for j in range(12)]
    with binding.Context(blob, max_slots=3, prefill=1, paged=1) as ctx:
        ctx.encode([a], [0])
        want = forced_logits(ctx, [0], [a], [toks], 1)[0]
        ctx.encode([b], [0])
        other = forced_logits(ctx, [0], [b], [toks], 1)[0]
        short = segments(shape, 2, 34, [4])[0]
        ctx.encode([a], [1])
        ctx.fork(1, [2])
        got = [ctx.decode_step([2], forced=[t], logits=True)[1][0] for t in toks[:5]]
        for t in toks:  # the source ends
            ctx.decode_step([1], forced=[t])
        ctx.encode([b], [1])  # its slot, another segment
        got_b = []
        for i, t in enumerate(toks):
            if i < 7:
                lg = ctx.decode_step([1, 2], forced=[t, toks[5 + i]], logits=True)[1]
                got.append(lg[1])
                if i == 3:
                    ctx.fork(2, [0])
            else:
                lg = ctx.decode_step([1], forced=[t], logits=True)[1]
            got_b.append(lg[0])
        assert np.array_equal(np.stack(got), want)
        assert np.array_equal(np.stack(got_b), other)
        last = [ctx.decode_step([0], forced=[t], logits=True)[1][0] for t in toks[9:]]
        assert np.array_equal(np.stack(last), want[9:])
        kv = ctx.debug_copy(binding.T_CROSS_K, 0, (shape.n_dec, shape.n_head, 1500, 64))
        ctx.encode([a], [2])
        assert np.array_equal(kv, ctx.debug_copy(binding.T_CROSS_K, 2, kv.shape))
        del short


@pytest.mark.parametrize("name,paged", [("tiny", 0), ("tiny", 1), ("base", 0)])
def test_drawn_tokens_follow_the_logits(name, paged):
    """Every drawn token is the choice, in float64, from the logits that a
    second slot returns when it is fed the drawn tokens; the filters hold."""
    shape, W, blob = model(name, n_enc=1, n_dec=2)
    segs = segments(shape, 10, 35)
    r = np.random.RandomState(4)
    sup, first = list(range(100, 160)), list(range(0, 50))
    opts = [dict(temperature=1.0, top_p=0.9), dict(temperature=0.7, top_k=40), dict(temperature=0.0),
            dict(temperature=1.4, top_k=100, top_p=0.95, min_p=0.01)]
    with binding.Context(blob, max_slots=8, paged=paged, prefill=1) as ctx:
        ctx.set_decoding(suppress=sup, suppress_first=first)
        ctx.encode(segs, [0, 1, 2, 3])
        ctx.encode(segs, [4, 5, 6, 7])
        for step in range(10):
            u = r.rand(4).astype(np.float32)
            kw = {k: [o.get(k, d) for o in opts] for k, d in
                  (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))}
            tok, lp = ctx.decode_sample([0, 1, 2, 3], u, **kw)
            _, lg = ctx.decode_step([4, 5, 6, 7], forced=tok, logits=True)
            for k, o in enumerate(opts):
                l = lg[k].astype(np.float64)
                l[sup] = -np.inf
                if step == 0:
                    l[first] = -np.inf
                f = lambda n, d: float(np.float32(o.get(n, d)))
                t, want = choose(l, float(u[k]), f("temperature", 1.0), o.get("top_k", 0), f("top_p", 1.0), f("min_p", 0.0))
                assert tok[k] == t, (step, k)
                assert abs(lp[k] - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -22 + 100 * 2.0 ** -24
        for k in range(4):
            assert np.array_equal(ctx.slot_tokens(k), [ctx.slot_tokens(k)[j] for j in range(10)])


def test_temperature_zero_is_the_greedy_step():
    shape, W, blob = model("tiny", n_enc=1, n_dec=2)
    segs = segments(shape, 7, 36, [3, 1, 5])
    with binding.Context(blob, max_slots=3) as ctx:
        ctx.encode(segs, [0, 1, 2])
        want = [[], [], []]
        for _ in range(20):
            act = [s for s in range(3) if len(want[s]) < len(segs[s].prompt) - 1 + 7]
            if act:
                for s, t in zip(act, ctx.decode_step(act)):
                    want[s].append(int(t))
        ctx.encode(segs, [0, 1, 2])
        got = [[], [], []]
        for _ in range(20):
            act = [s for s in range(3) if len(got[s]) < len(segs[s].prompt) - 1 + 7]
            if act:
                tok, lp = ctx.decode_sample(act, np.full(len(act), 0.77), temperature=0.0)
                assert all((l == 0) == (t < 0) for l, t in zip(lp, tok))
                for s, t in zip(act, tok):
                    got[s].append(int(t))
    assert got == want


@pytest.mark.parametrize("paged", [0, 1])
def test_drawn_steps_are_profiled(paged):
    shape, W, blob = model("tiny")
    segs = segments(shape, 8, 36, [3, 3])
    with binding.Context(blob, max_slots=2, prefill=1, paged=paged) as ctx:
        ctx.encode(segs, [0, 1])
        ctx.profile_enable(binding.K_DEC_STEP, True)
        for _ in range(3):
            ctx.decode_sample([0, 1], [0.2, 0.9])
        ms, n = ctx.profile_read(binding.K_DEC_STEP)
        assert n == 3 and ms > 0


def test_allocation_free_steps_of_forks():
    torch = pytest.importorskip("torch")
    shape, W, blob = model("base", n_enc=1, n_dec=2)
    seg = segments(shape, 8, 37, [66])[0]
    out = torch.zeros(3, dtype=torch.int32, device="cuda")
    with binding.Context(blob, max_slots=4, prefill=1, paged=1) as ctx:
        want = ctx.transcribe([seg])[0]["tokens"]
        ctx.encode([seg], [1])
        ctx.decode_step_noalloc([1])
        ctx.fork(1, [3, 0])
        got = []
        for _ in range(7):
            ctx.decode_step_noalloc([0, 3, 1], out.data_ptr())
            torch.cuda.synchronize()
            ctx.stats()
            got.append(out.cpu().numpy().copy())
        assert (np.stack(got) == want[1:, None]).all()
        assert np.array_equal(ctx.slot_tokens(0), want)


def test_recorded_step_of_a_later_fork():
    """A recorded allocation-free step, replayed when its slot has become the
    fork of another and then past the tokens it reserved, reads the caches that
    the slot has by then and leaves the other slots' pages alone."""
    torch = pytest.importorskip("torch")
    shape, W, blob = model("base", n_enc=1, n_dec=2)
    a, b = segments(shape, 30, 40, [40, 40])
    b.audio = a.audio[::-1].copy()
    b.max_new_tokens = 1
    with binding.Context(blob, max_slots=3, prefill=1, paged=1) as ctx:
        want, other = (ctx.transcribe([s])[0]["tokens"] for s in (a, b))
        st = torch.cuda.Stream()
        ctx.set_stream(st.cuda_stream)
        out = torch.full((1,), -7, dtype=torch.int32, device="cuda")
        ctx.encode([a], [0])
        ctx.encode([b], [1])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            ctx.decode_step_noalloc([1], out.data_ptr())
        g.replay()
        torch.cuda.synchronize()
        assert out.item() == other[0]
        # slot 1 has its one token and is idle
        ctx.fork(0, [1])
        ctx.encode([b], [2])
        for step in range(100):  # positions 39 .. 138: the fork holds 70, in two pages of 64
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            if step < 30:
                assert out.item() == want[step], step
        got = [ctx.decode_step([0])[0] for _ in range(30)]
        assert np.array_equal(np.ravel(got), want)


def test_best_of_five():
    """As a program uses them: a segment's prompt prefilled once, five
    candidates drawn, the likeliest kept; its log-probability is the oracle's."""
    from oracle import model as M
    import oracle
    shape, W, blob = model("tiny")
    seg = segments(shape, 12, 38, [20])[0]
    r = np.random.RandomState(6)
    slots = [0, 1, 2, 3, 4]
    with binding.Context(blob, max_slots=5, prefill=1, paged=1) as ctx:
        ctx.set_decoding(suppress=[3, 4, 5])
        ctx.encode([seg], [0])
        ctx.fork(0, slots[1:])
        score = np.zeros(5)
        for _ in range(12):
            tok, lp = ctx.decode_sample(slots, r.rand(5), temperature=0.8, top_p=0.95)
            score += lp
        best = int(np.argmax(score))
        tokens = ctx.slot_tokens(best)
        drawn = {tuple(ctx.slot_tokens(s)) for s in slots}
    assert len(drawn) > 1 and tokens.size == 12 and not set(tokens) & {3, 4, 5}
    E = M.encoder(W, shape, oracle.log_mel_segment(seg.audio, shape.n_mels)[None])
    ckv = M._seg_ckv(M.cross_kv(W, shape, E), 0)
    lg = np.array(M.greedy(W, shape, ckv, list(seg.prompt), 12, forced=[int(t) for t in tokens])[1])
    lg[:, [3, 4, 5]] = -np.inf
    want = 0.0
    for l, t in zip(lg, tokens):
        want += l[t] - l.max() - np.log(np.exp(l - l.max()).sum())
    # every logit within the fp32 model's tolerance of its row's largest: so is a log-probability, twice
    assert abs(score[best] - want) <= 12 * 2 * TOL["f32"] * np.abs(lg[np.isfinite(lg)]).max()


def test_refusals():
    shape, W, blob = model("tiny", n_enc=1, n_dec=1)
    seg = segments(shape, 3, 39, [2])[0]

    def refused(status, f, *a, **kw):
        with pytest.raises(binding.WhisperError) as e:
            f(*a, **kw)
        assert e.value.status == status, e.value

    with binding.Context(blob, max_slots=2) as ctx:
        ctx.encode([seg], [0])
        refused(binding.E_STATE, ctx.fork, 0, [1])
    with binding.Context(blob, max_slots=3, paged=1) as ctx:
        ctx.encode([seg], [0])
        refused(binding.E_STATE, ctx.fork, 1, [2])
        refused(binding.E_STATE, ctx.fork, 0, [0])
        refused(binding.E_INVAL, ctx.fork, 0, [1, 1])
        refused(binding.E_CAPACITY, ctx.fork, 0, [3])
        refused(binding.E_CAPACITY, ctx.fork, 3, [1])
        refused(binding.E_STATE, ctx.decode_sample, [1], [0.5])
        refused(binding.E_INVAL, ctx.decode_sample, [0], [0.5], top_p=0.0)
        refused(binding.E_INVAL, ctx.decode_sample, [0, 0], [0.5, 0.5])
        refused(binding.E_INVAL, ctx.decode_sample, [0], [0.5, 0.5])
        refused(binding.E_CAPACITY, ctx.decode_sample, [5], [0.5])
        ctx.fork(0, [])
        ctx.fork(0, [2])
        assert ctx.decode_step([0])[0] == -1
        assert ctx.decode_step([0, 2])[1] == -1
    p = binding.params_from_blob(blob)
    assert p.paged == 0


def record(torch, ctx, slots, out, steps=1):
    """A stream for the context, and a graph of allocation-free steps on it."""
    st = torch.cuda.Stream()
    ctx.set_stream(st.cuda_stream)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        for _ in range(steps):
            ctx.decode_step_noalloc(slots, out.data_ptr())
    return st, g


def replay(torch, g, n, out=None):
    got = []
    for _ in range(n):
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        if out is not None:
            got.append(out.cpu().numpy().copy())
    return got


@pytest.mark.parametrize("paged", [0, 1])
def test_replays_past_the_text_context(paged):
    """A recorded step that is replayed beyond position 447 leaves the other
    slots' tokens, prompts and caches alone: an idle neighbour's seated prompt,
    a half-decoded neighbour's first positions, and what lies behind the last slot."""
    torch = pytest.importorskip("torch")
    shape, W, blob = model("base", n_enc=1, n_dec=2)
    full = segments(shape, 444, 44, [4, 4, 4])
    near = segments(shape, 30, 45, [6, 6])
    out = torch.full((3,), -7, dtype=torch.int32, device="cuda")
    with binding.Context(blob, max_slots=5, paged=paged) as ctx:
        want = [r["tokens"] for r in ctx.transcribe(full + near)]
        ctx.encode([full[0], near[0], full[1], near[1], full[2]], [0, 1, 2, 3, 4])
        for _ in range(7):
            ctx.decode_step([3])
        st, g = record(torch, ctx, [0, 2, 4], out)
        got = np.stack(replay(torch, g, 470, out))
        assert (got[:3] == -1).all()
        for k in range(3):
            assert np.array_equal(got[3: 447, k], want[k])
        tail = [ctx.decode_step([1])[0] for _ in range(35)][5:]
        assert np.array_equal(tail, want[3])
        tail = [ctx.decode_step([3])[0] for _ in range(28)]
        assert np.array_equal(tail, want[4][2:])


@pytest.mark.parametrize("name", ["tiny", "base"])
def test_fork_of_a_slot_that_replays_moved_on(name):
    """Replays move a slot on the device alone: a fork is made where the slot
    stands there, and the calls' counts follow."""
    torch = pytest.importorskip("torch")
    shape, W, blob = model(name, n_enc=1, n_dec=2)
    seg = segments(shape, 150, 42, [5])[0]
    out = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    with binding.Context(blob, max_slots=4, prefill=1, paged=1) as ctx:
        want = ctx.transcribe([seg])[0]["tokens"]
        other = segments(shape, 140, 43, [300])[0]
        for _ in range(2):  # pages that hold something else's keys
            ctx.encode([other] * 4, [0, 1, 2, 3])
            for _ in range(140):
                ctx.decode_step([0, 1, 2, 3])
        ctx.encode([seg], [0])
        st, g = record(torch, ctx, [0], out)
        got = replay(torch, g, 81, out)
        assert np.array_equal(np.ravel(got), want[:81])
        ctx.fork(0, [1, 3])
        for s in (0, 1, 3):
            assert np.array_equal(ctx.slot_tokens(s), want[:81])
        rest = [ctx.decode_step([3, 0, 1]) for _ in range(69)]
        assert (np.stack(rest) == want[81:, None]).all()
        for s in (0, 1, 3):  # all 150: idle
            assert np.array_equal(ctx.slot_tokens(s), want)
            with pytest.raises(binding.WhisperError) as e:
                ctx.decode_step([s])
            assert e.value.status == binding.E_STATE
        # recorded steps that never ran: the device is where the encode left it
        ctx.encode([seg], [0])
        st, g = record(torch, ctx, [0], out, steps=70)
        ctx.fork(0, [2])
        assert ctx.slot_tokens(0).size == 0 and ctx.slot_tokens(2).size == 0
        rest = [ctx.decode_step([2, 0]) for _ in range(150)]
        assert (np.stack(rest) == want[:, None]).all()
        # inside the prompt, and past the last token
        ctx.encode([seg], [1])
        st, g = record(torch, ctx, [1], out)
        replay(torch, g, 150)
        with pytest.raises(binding.WhisperError) as e:
            ctx.fork(1, [3])
        assert e.value.status == binding.E_STATE
    with binding.Context(blob, max_slots=2, paged=1) as ctx:
        ctx.encode([seg], [0])
        st, g = record(torch, ctx, [0], out)
        assert [int(x[0]) for x in replay(torch, g, 3, out)] == [-1, -1, -1]
        ctx.fork(0, [1])
        assert [ctx.decode_step([0, 1]).tolist() for _ in range(3)] == [[-1, -1], [want[0]] * 2, [want[1]] * 2]


def drawn_steps(ctx, slots, n, seed):
    r = np.random.RandomState(seed)
    return [ctx.decode_sample(slots, r.rand(len(slots)), temperature=1.0, top_p=0.95) for _ in range(n)]


@pytest.mark.parametrize("paged", [0, 1])
def test_drawn_tokens_are_the_slots_tokens(paged):
    """slot_tokens returns what the drawn steps returned, and the next step's
    input is the drawn token."""
    shape, W, blob = model("tiny", n_enc=1, n_dec=2)
    segs = segments(shape, 10, 41)
    with binding.Context(blob, max_slots=8, paged=paged, prefill=1) as ctx:
        ctx.encode(segs, [0, 1, 2, 3])
        drawn = [t for t, _ in drawn_steps(ctx, [0, 1, 2, 3], 9, 5)]
        ctx.encode(segs, [4, 5, 6, 7])
        for t in drawn:
            ctx.decode_step([4, 5, 6, 7], forced=t)
        last, logits = ctx.decode_step([0, 1, 2, 3, 4, 5, 6, 7], logits=True)
        assert np.array_equal(logits[:4], logits[4:])
        for k in range(4):
            assert np.array_equal(ctx.slot_tokens(k), [t[k] for t in drawn] + [last[k]])


def test_draws_and_forks_refuse_a_recording_stream():
    """They wait for the device, which would end the recording: refused, and the
    recording, the context and its slots go on."""
    torch = pytest.importorskip("torch")
    shape, W, blob = model("tiny", n_enc=1, n_dec=2)
    seg = segments(shape, 6, 46, [4])[0]
    out = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    with binding.Context(blob, max_slots=3, prefill=1, paged=1) as ctx:
        want = ctx.transcribe([seg])[0]["tokens"]
        ctx.encode([seg, seg], [0, 1])
        st = torch.cuda.Stream()
        ctx.set_stream(st.cuda_stream)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            ctx.decode_step_noalloc([0], out.data_ptr())
            for f in (lambda: ctx.decode_sample([1], [0.5]), lambda: ctx.fork(1, [2])):
                with pytest.raises(binding.WhisperError) as e:
                    f()
                assert e.value.status == binding.E_STATE
        got = replay(torch, g, 2, out)
        assert np.array_equal(np.ravel(got), want[:2])
        ctx.fork(0, [2])
        assert ctx.decode_sample([2, 1], [0.5, 0.5], temperature=0.0)[0].tolist() == [want[2], want[0]]
