"""Operators of beam search over a packed key/value cache.

A recogniser that searches with several beams per utterance holds as many
sequences as beams, so its cache is what limits the batch. These cases are of a
cache whose keys and values are kept in 8 or 4 bits, and of the search's own
steps. Each case is one of

* op "store": the keys and values of `n` sequences' new tokens (1 .. `new`
  each), all layers, are quantised behind what the sequences hold, and the
  sequences read back;
* op "attend": causal attention of `n` sequences' new tokens over `past` cached
  positions at most and themselves, the cache packed;
* op "beam": the `best` likeliest continuations of every group of `width`
  beams, from the beams' scores and their rows of `vocab` logits;
* op "reorder": sequences become copies of the chosen beams' sequences (all at
  once), one token is appended to each, and they are read out.

What a packed cache stands for: 64 numbers of a row form a group. With lo and hi
their least and largest, 0 included, the step is the smallest number with four
(8 bits: one) significant bits that is at least (hi - lo) / 15 (255), and at
least 2^-100; zero = round(-lo / step); code = round(x / step) + zero, in 0 .. 15
(255); the value is (code - zero) * step. Halves round to even. It is exact in
bf16 and in fp32.
"""
import math

import numpy as np
import torch

own = False


def listed():
    def attend(name, dtype, bits, n, past, new, heads, kv_heads, size, page):
        return {"name": name, "op": "attend", "dtype": dtype, "bits": bits, "n": n, "past": past, "new": new,
                "heads": heads, "kv_heads": kv_heads, "size": size, "page": page}

    def store(name, dtype, bits, n, past, new, layers, kv_heads, size, page):
        return {"name": name, "op": "store", "dtype": dtype, "bits": bits, "n": n, "past": past, "new": new,
                "layers": layers, "kv_heads": kv_heads, "size": size, "page": page}

    def beam(name, dtype, groups, width, best, vocab):
        return {"name": name, "op": "beam", "dtype": dtype, "groups": groups, "width": width, "best": best,
                "vocab": vocab}

    def reorder(name, dtype, bits, groups, width, past, layers, kv_heads, size, page):
        return {"name": name, "op": "reorder", "dtype": dtype, "bits": bits, "groups": groups, "width": width,
                "past": past, "layers": layers, "kv_heads": kv_heads, "size": size, "page": page}

    return [
        # one step of one utterance on the smallest fp32 model: latency
        attend("attend4-f32-step-1", "f32", 4, 1, 37, 1, 6, 6, 64, 64),
        # one step of a full batch of the largest model, ragged
        attend("attend4-step-32", "bf16", 4, 32, 447, 1, 20, 20, 64, 64),
        # few rows over long contexts, grouped heads: the cache's bytes
        attend("attend4-long-4", "bf16", 4, 4, 60001, 1, 32, 8, 128, 128),
        # five drafted tokens per sequence to verify in one pass, 8 bits
        attend("attend8-draft-16", "bf16", 8, 16, 4001, 5, 16, 4, 64, 32),
        # a long document's next chunk: the matrix cores
        attend("attend4-fill-4096", "bf16", 4, 1, 4097, 4096, 32, 8, 128, 64),
        # prompts quantised behind earlier text, a small model's layers
        store("store4-prompts-16", "bf16", 4, 16, 101, 224, 12, 12, 64, 32),
        # a decode step's keys and values, every layer of the largest model, 8 bits
        store("store8-step-32", "bf16", 8, 32, 20, 1, 32, 20, 64, 64),
        # one utterance's five beams
        beam("beam-1x5", "f32", 1, 5, 10, 51865),
        # a batch of utterances, some at their first step
        beam("beam-64x5", "bf16", 64, 5, 10, 51866),
        # wide beams over a wide vocabulary
        beam("beam-16x12", "f32", 16, 12, 24, 151937),
        # one utterance's beams on the smallest model, cache not packed: latency
        reorder("reorder-f32-1x5", "f32", 0, 1, 5, 37, 4, 6, 64, 64),
        # a batch's beams after a step, every layer of the largest model
        reorder("reorder4-8x5", "bf16", 4, 8, 5, 61, 32, 20, 64, 64),
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "store", "beam", "beam", "reorder"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "beam":
        vocab, width = _log(rng, 33, 152000), rng.choice([1, 2, 3, 4, 5, 6, 8, 10, 12, 16])
        most = max(1, min(512, 20000000 // vocab) // width)
        return {"op": op, "dtype": dtype, "groups": _log(rng, 1, most), "width": width,
                "best": rng.choice([width, 2 * width, 2 * width]), "vocab": vocab}
    bits = rng.choice([4, 4, 8])
    page = rng.choice([32, 64, 128])
    size = rng.choice([64, 64, 128])
    kv = rng.choice([1, 2, 4, 5, 8, 12, 16, 20])
    if op == "reorder":
        layers, groups, width = rng.choice([1, 4, 6, 12, 24, 32]), _log(rng, 1, 16), rng.choice([2, 3, 4, 5, 6, 8])
        top = max(2, 100000000 // (layers * kv * size * groups * width))
        return {"op": op, "dtype": dtype, "bits": rng.choice([0, 4, 4, 8]), "groups": groups, "width": width,
                "past": _log(rng, 1, min(2000, top)), "layers": layers, "kv_heads": kv, "size": size, "page": page}
    if op == "store":
        layers, n = rng.choice([1, 4, 6, 12, 24, 32]), _log(rng, 1, 16)
        top = max(2, 100000000 // (layers * kv * size * n))  # positions per sequence
        return {"op": op, "dtype": dtype, "bits": bits, "n": n, "past": _log(rng, 1, min(2000, top)),
                "new": rng.choice([1, _log(rng, 1, min(1000, top))]), "layers": layers, "kv_heads": kv, "size": size,
                "page": page}
    group = rng.choice([1, 1, 2, 4, 5, 8])
    while group * kv > 40:
        group = rng.choice([1, 2])
    kind = rng.choice(["step", "step", "draft", "prompts"])
    new = {"step": 1, "draft": rng.randint(2, 8), "prompts": _log(rng, 9, 1500)}[kind]
    n = _log(rng, 1, {"step": 64, "draft": 32, "prompts": 16}[kind])
    cells = 200000000 if dtype == "bf16" else 60000000  # scores of one pass, and the cached numbers
    past = min(60000, max(1, cells // (n * new * kv * group)), max(1, cells // (n * kv * size)))
    return {"op": op, "dtype": dtype, "bits": bits, "n": n, "past": _log(rng, 1, past), "new": new, "heads": kv * group,
            "kv_heads": kv, "size": size, "page": page}


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[case["dtype"]]


def _lengths(case):
    """Cached positions and new tokens of every sequence, the same for every
    seed: the first has the case's, the others a ragged share of them."""
    n, past, new = case["n"], case["past"], case["new"]
    r = np.random.RandomState(n * 1013 + past)
    p = [past] + [int(x) for x in r.randint(past // 16, past + 1, n - 1)]
    c = [new] + [int(x) for x in r.randint((new + 3) // 4, new + 1, n - 1)]
    return p, c


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(gen, shape, dtype):
    """Keys or values: some numbers of every head are larger than the others in all rows."""
    x = torch.randn(shape, generator=gen, device="cuda")
    x[..., 5::23] *= 3
    return x.to(dtype)


def _attend_inputs(case, seed):
    past, new = _lengths(case)
    g, t = _generator(seed), _dtype(case)
    kv, size = case["kv_heads"], case["size"]
    k = [_rows(g, (p + c, kv, size), t) for p, c in zip(past, new)]
    v = [_rows(g, (p + c, kv, size), t) for p, c in zip(past, new)]
    q = (torch.randn((sum(new), case["heads"], size), generator=g, device="cuda") * 1.2).to(t)
    return past, new, q, k, v


def _store_inputs(case, seed):
    past, new = _lengths(case)
    g, t = _generator(seed), _dtype(case)
    shape = (case["kv_heads"], case["size"])
    old = [[_rows(g, (case["layers"], p, *shape), t) for p in past] for _ in range(2)]
    k, v = (_rows(g, (case["layers"], sum(new), *shape), t) for _ in range(2))
    return past, new, old, k, v


def _reorder_inputs(case, seed):
    g, t = _generator(seed), _dtype(case)
    n = case["groups"] * case["width"]
    shape = (case["kv_heads"], case["size"])
    old = [[_rows(g, (case["layers"], case["past"], *shape), t) for _ in range(n)] for _ in range(2)]
    k, v = (_rows(g, (case["layers"], n, *shape), t) for _ in range(2))
    r = np.random.RandomState(seed % 2**31)
    parents = [b // case["width"] * case["width"] + int(r.randint(case["width"])) for b in range(n)]
    return old, k, v, parents


def _live(case):
    """Beams of every group: every eighth group is at its first step and has one."""
    return [1 if g % 8 == 7 else case["width"] for g in range(case["groups"])]


def _beam_inputs(case, seed):
    g = _generator(seed)
    r = np.random.RandomState(seed % 2**31)
    W, V = case["width"], case["vocab"]
    rows = case["groups"] * W
    logits = torch.randn((rows, V), generator=g, device="cuda") * 2.5
    likely = torch.randint(0, V, (rows, 5), generator=g, device="cuda")
    logits.scatter_add_(1, likely, torch.rand((rows, 5), generator=g, device="cuda") * 14)
    # a range of ids ruled out by the program in every third row (timestamps before the last one)
    logits[::3, V - V // 34:] = -math.inf
    scores = torch.rand(rows, generator=g, device="cuda") * -20
    for i, n in enumerate(_live(case)):
        scores[i * W + n: (i + 1) * W] = -math.inf
    suppress = np.unique(r.randint(0, V, min(88, V // 8))).astype(np.int32)  # never chosen, as set once for a model
    return logits.to(_dtype(case)), scores, suppress


# ------------------------------------------------------------------ a packed cache, plain

def _pack(x, bits):
    """Codes of rows x [...][size] (two a byte in 4 bits), steps and zeros [...][size / 64]."""
    top, low = (15, 20) if bits == 4 else (255, 23)  # mantissa bits that a step lacks
    g = x.float().unflatten(-1, (-1, 64))
    lo, hi = g.amin(-1).clamp(max=0), g.amax(-1).clamp(min=0)
    step = ((hi - lo).double() / top).float()  # (a quotient just above a step would be taken for it)
    step = (step.view(torch.int32) + ((1 << low) - 1) >> low << low).view(torch.float32).clamp(min=2.0**-100)
    zero = torch.round(-lo / step)
    code = (torch.round(g / step[..., None]) + zero[..., None]).clamp(0, top).to(torch.uint8).flatten(-2)
    if bits == 4:
        code = code[..., 0::2] | code[..., 1::2] << 4
    return code, step, zero


def _unpack(code, step, zero, bits):
    """Their values in fp32."""
    if bits == 4:
        code = torch.stack([code & 15, code >> 4], -1).flatten(-2)
    return ((code.float().unflatten(-1, (-1, 64)) - zero[..., None]) * step[..., None]).flatten(-2)


class _Pages:
    """Keys or values as [layer][page][position][head] rows: as they are (bits 0) or packed."""

    def __init__(self, layers, count, page, kv, size, bits, dtype):
        self.page, self.bits, self.dtype = page, bits, dtype
        at = (layers, count, page, kv)
        if bits:
            self.parts = [torch.zeros((*at, size * bits // 8), dtype=torch.uint8, device="cuda"),
                          *(torch.zeros((*at, size // 64), device="cuda") for _ in range(2))]
        else:
            self.parts = [torch.zeros((*at, size), dtype=dtype, device="cuda")]

    def put(self, pages, first, rows):
        """rows [layer][n][head][size] from position `first` of the sequence whose pages are given."""
        at = torch.arange(first, first + rows.shape[1], device="cuda")
        where = pages[at // self.page]
        for p, x in zip(self.parts, _pack(rows, self.bits) if self.bits else [rows]):
            p[:, where, at % self.page] = x

    def get(self, pages, n):
        """The first n positions [layer][n][head][size]: fp32 if packed."""
        got = [p[:, pages].flatten(1, 2)[:, :n] for p in self.parts]
        return _unpack(*got, self.bits) if self.bits else got[0]

    def copy(self, src, dst):
        for p in self.parts:
            p[:, dst] = p[:, src]


def _ids(x):
    return torch.tensor(x, dtype=torch.long, device="cuda")


# ------------------------------------------------------------------ preparation

def _cache(case, layers, kv, lens, n_pages, heads=None):
    """The framework's cache for sequences of up to lens positions."""
    from paper_2507_01021_amd import binding
    c = binding.Cache(dtype=binding.DTYPE_F32 if case["dtype"] == "f32" else binding.DTYPE_BF16, n_layer=layers,
                      n_head=heads or kv, n_kv_head=kv, head_size=case["size"], page_size=case["page"],
                      n_pages=n_pages, max_seqs=len(lens), max_positions=max(lens), max_tokens=sum(lens),
                      bits=case["bits"])
    c.set_stream(torch.cuda.current_stream().cuda_stream)
    return c


def prepare(case, seed):
    st = {"case": case}
    return {"beam": _prepare_beam, "attend": _prepare_attend, "store": _prepare_store,
            "reorder": _prepare_reorder}[case["op"]](st, case, seed)


def _prepare_beam(st, case, seed):
    st["logits"], st["scores"], suppress = _beam_inputs(case, seed)
    G, W, n = case["groups"], case["width"], case["best"]
    if own:
        from paper_2507_01021_amd import binding
        b = binding.Beam(case["vocab"], G * W)
        b.set_stream(torch.cuda.current_stream().cuda_stream)
        b.options(suppress=suppress)
        st["beam"] = b
        st["dt"] = binding.DTYPE_F32 if case["dtype"] == "f32" else binding.DTYPE_BF16
        st["parents"], st["tokens"] = (torch.empty((G, n), dtype=torch.int32, device="cuda") for _ in range(2))
        st["out"] = torch.empty((G, n), dtype=torch.float32, device="cuda")
    else:
        st["suppress"] = torch.from_numpy(suppress.astype(np.int64)).cuda()
    return st


def _prepare_attend(st, case, seed):
    P, kv, size = case["page"], case["kv_heads"], case["size"]
    past, new, q, k, v = _attend_inputs(case, seed)
    n, lens = len(past), [p + c for p, c in zip(past, new)]
    count = sum(-(-x // P) for x in lens)
    st["q"], st["new"], st["past"] = q, new, past
    if own:
        c = _cache(case, 1, kv, lens, count, case["heads"])
        some = [s for s in range(n) if past[s]]
        for seqs, lo, hi in ((some, [0] * n, past), (list(range(n)), past, lens)):
            if not seqs:
                continue
            kk, vv = (torch.cat([x[s][lo[s]:hi[s]] for s in seqs]) for x in (k, v))
            c.extend(seqs, [hi[s] - lo[s] for s in seqs])
            c.append(0, kk.data_ptr(), vv.data_ptr())
            torch.cuda.synchronize()
        st["cache"] = c
        st["out"] = torch.empty_like(q)
    else:
        free = [int(x) for x in np.random.RandomState(seed % 2**31).permutation(count)]
        st["pages"] = [_ids([free.pop() for _ in range(-(-x // P))]) for x in lens]
        st["k"], st["v"] = (_Pages(1, count, P, kv, size, case["bits"], _dtype(case)) for _ in range(2))
        for pages, rows in ((st["k"], k), (st["v"], v)):
            for s in range(n):
                pages.put(st["pages"][s], 0, rows[s][None])
    return st


def _prepare_store(st, case, seed):
    P, kv, size, L, t = case["page"], case["kv_heads"], case["size"], case["layers"], _dtype(case)
    past, new, old, st["nk"], st["nv"] = _store_inputs(case, seed)
    ends = [p + c for p, c in zip(past, new)]
    count = sum(-(-x // P) for x in ends)
    st["past"], st["new"], st["ends"] = past, new, ends
    st["k_out"], st["v_out"] = (torch.empty((L, sum(ends), kv, size), dtype=t, device="cuda") for _ in range(2))
    if own:
        c = _cache(case, L, kv, ends, count)
        some = [s for s in range(len(past)) if past[s]]
        if some:
            kk, vv = (torch.cat([x[s] for s in some], 1) for x in old)
            c.extend(some, [past[s] for s in some])
            c.append(-1, kk.data_ptr(), vv.data_ptr())
            torch.cuda.synchronize()
        st["cache"] = c
    else:
        free = list(range(count - 1, -1, -1))
        st["pages"] = [_ids([free.pop() for _ in range(-(-x // P))]) for x in ends]
        st["k"], st["v"] = (_Pages(L, count, P, kv, size, case["bits"], t) for _ in range(2))
        for pages, rows in ((st["k"], old[0]), (st["v"], old[1])):
            for s, r in enumerate(rows):
                if past[s]:
                    pages.put(st["pages"][s], 0, r)
    return st


def _prepare_reorder(st, case, seed):
    P, kv, size, L, t = case["page"], case["kv_heads"], case["size"], case["layers"], _dtype(case)
    old, st["nk"], st["nv"], st["parents"] = _reorder_inputs(case, seed)
    n, past = len(st["parents"]), case["past"]
    per = -(-past // P)
    count = n * (per + 2)  # the beams, and a page or two of its own for every new one
    st["k_out"], st["v_out"] = (torch.empty((L, n * (past + 1), kv, size), dtype=t, device="cuda") for _ in range(2))
    if own:
        c = _cache(case, L, kv, [past] * n + [past + 1] * n, count)
        kk, vv = (torch.cat(x, 1) for x in old)
        c.extend(list(range(n)), [past] * n)
        c.append(-1, kk.data_ptr(), vv.data_ptr())
        torch.cuda.synchronize()
        st["cache"] = c
    else:
        st["k"], st["v"] = (_Pages(L, count, P, kv, size, case["bits"], t) for _ in range(2))
        st["pages"] = [list(range(s * per, (s + 1) * per)) for s in range(n)]
        for pages, rows in ((st["k"], old[0]), (st["v"], old[1])):
            for s, r in enumerate(rows):
                pages.put(_ids(st["pages"][s]), 0, r)
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    return {"beam": _run_beam, "attend": _run_attend, "store": _run_store, "reorder": _run_reorder}[st["case"]["op"]](st)


def _run_beam(st):
    case = st["case"]
    G, W, V, n = case["groups"], case["width"], case["vocab"], case["best"]
    if own:
        st["beam"].run(st["logits"].data_ptr(), st["dt"], G, W, n, st["scores"].data_ptr(), st["parents"].data_ptr(),
                       st["tokens"].data_ptr(), st["out"].data_ptr())
        return st["parents"], st["tokens"], st["out"]
    # in 64 bits: scores next to each other decide which is chosen
    l = st["logits"].double()
    l[:, st["suppress"]] = -math.inf
    m = l.amax(1, keepdim=True)
    l -= m + torch.exp(l - m).sum(1, keepdim=True).log()
    l += st["scores"].double()[:, None]
    best = torch.sort(l.view(G, W * V), dim=1, descending=True, stable=True)
    at, score = best.indices[:, :n], best.values[:, :n]
    none = score == -math.inf
    return (at // V).masked_fill(none, -1).int(), (at % V).masked_fill(none, -1).int(), score.float()


def _run_attend(st):
    case, q = st["case"], st["q"]
    if own:
        st["cache"].attend(0, q.data_ptr(), st["out"].data_ptr())
        return st["out"]
    H, kv, D = case["heads"], case["kv_heads"], case["size"]
    G = H // kv
    out = torch.empty_like(q)
    r = 0
    for s, (p, c) in enumerate(zip(st["past"], st["new"])):
        k, v = (x.get(st["pages"][s], p + c)[0] for x in (st["k"], st["v"]))
        hidden = torch.arange(p + c, device="cuda")[None, :] > torch.arange(p, p + c, device="cuda")[:, None]
        x = q[r: r + c].float().transpose(0, 1).reshape(kv, G * c, D)
        a = torch.matmul(x, k.permute(1, 2, 0).contiguous()) / math.sqrt(D)
        a = a.view(H, c, p + c).masked_fill_(hidden, -math.inf)
        a = torch.exp(a - a.amax(-1, keepdim=True))
        a = (a / a.sum(-1, keepdim=True)).view(kv, G * c, p + c)
        y = torch.matmul(a, v.transpose(0, 1).contiguous())
        out[r: r + c] = y.view(H, c, D).transpose(0, 1).to(q.dtype)
        r += c
    return out


def _read(st, pages, ends):
    at = 0
    for where, n in zip(pages, ends):
        for x, out in ((st["k"], st["k_out"]), (st["v"], st["v_out"])):
            out[:, at: at + n] = x.get(where, n).to(out.dtype)
        at += n
    return st["k_out"], st["v_out"]


def _run_store(st):
    seqs = list(range(len(st["past"])))
    if own:
        c = st["cache"]
        c.truncate(seqs, st["past"])
        c.extend(seqs, st["new"])
        c.append(-1, st["nk"].data_ptr(), st["nv"].data_ptr())
        c.read(-1, seqs, st["k_out"].data_ptr(), st["v_out"].data_ptr())
        return st["k_out"], st["v_out"]
    r = 0
    for s in seqs:
        for x, rows in ((st["k"], st["nk"]), (st["v"], st["nv"])):
            x.put(st["pages"][s], st["past"][s], rows[:, r: r + st["new"][s]])
        r += st["new"][s]
    return _read(st, st["pages"], st["ends"])


def _run_reorder(st):
    case, parents = st["case"], st["parents"]
    n, past, P = len(parents), case["past"], case["page"]
    if own:
        c, new = st["cache"], list(range(n, 2 * n))
        c.reorder(new, parents)
        c.extend(new, [1] * n)
        c.append(-1, st["nk"].data_ptr(), st["nv"].data_ptr())
        c.read(-1, new, st["k_out"].data_ptr(), st["v_out"].data_ptr())
        return st["k_out"], st["v_out"]
    # whole pages are shared, a partly filled one is copied
    per, full = -(-past // P), past // P
    lists = []
    for i, b in enumerate(parents):
        pages, mine = st["pages"][b][:full], n * per + i
        if past % P:
            for x in (st["k"], st["v"]):
                x.copy(st["pages"][b][full], mine)
        lists.append(_ids(pages + [mine]))
        for x, rows in ((st["k"], st["nk"]), (st["v"], st["nv"])):
            x.put(lists[-1], past, rows[:, i: i + 1])
    return _read(st, lists, [past + 1] * n)


# ------------------------------------------------------------------ work and exact results

def _row_bytes(case):
    """A head's row in the caller's type, and as the cache holds it."""
    b = 4 if case["dtype"] == "f32" else 2
    D, bits = case["size"], case["bits"]
    return D * b, D * bits // 8 + D // 64 * 2 if bits else D * b


def work(case):
    op = case["op"]
    if op == "beam":
        b = 4 if case["dtype"] == "f32" else 2
        rows = sum(_live(case))
        return {"bytes": rows * (case["vocab"] * b + 4) + case["groups"] * case["best"] * 12,
                "flops": 4 * rows * case["vocab"]}
    kv, D = case["kv_heads"], case["size"]
    row, held = _row_bytes(case)
    if op == "reorder":  # beams read, new rows read and written, everything copied out
        n = case["groups"] * case["width"]
        return {"bytes": 2 * case["layers"] * kv * n * (case["past"] * held + row + held + (case["past"] + 1) * row),
                "flops": 0}
    past, new = _lengths(case)
    if op == "store":  # what was there is read and copied out; new rows are read, written and copied out
        return {"bytes": 2 * case["layers"] * kv * (sum(past) * (held + row) + sum(new) * (2 * row + held)), "flops": 0}
    H = case["heads"]
    return {"bytes": 2 * kv * held * (sum(past) + sum(new)) + 2 * H * row * sum(new),
            "flops": sum(4 * H * D * c * (p + (c + 1) / 2) for p, c in zip(past, new))}


def _held(x, bits):
    """What a cache of `bits` makes of rows x, in 64 bits."""
    x = x.double()
    if not bits:
        return x
    top = 2**bits - 1
    g = x.reshape(*x.shape[:-1], -1, 64)
    none = torch.zeros_like(g[..., 0])
    least, most = torch.minimum(none, g.min(-1).values), torch.maximum(none, g.max(-1).values)
    spread = (most - least).float().double()  # (a range is held in 32 bits)
    # (a plain number as divisor would be multiplied by its reciprocal, which is off where the quotient is a step
    # itself, and powers from torch.ldexp are off in the last place: quotient / fraction is exact)
    step = spread / torch.full_like(spread, top)
    frac = torch.frexp(step).mantissa
    digits = 2.0 ** (4 if bits == 4 else 1)
    step = torch.where(frac > 0, torch.ceil(frac * digits) / digits * (step / frac), step)
    step = torch.where(step < 2.0**-100, torch.full_like(step, 2.0**-100), step)
    zero = torch.round(-least / step)
    code = torch.round(g / step[..., None]) + zero[..., None]
    code = torch.minimum(torch.maximum(code, torch.zeros_like(code)), torch.full_like(code, top))
    return ((code - zero[..., None]) * step[..., None]).reshape(x.shape)


def exact(case, seed):
    return {"beam": _exact_beam, "attend": _exact_attend, "store": _exact_store,
            "reorder": _exact_reorder}[case["op"]](case, seed)


def _exact_attend(case, seed):
    past, new, q, k, v = _attend_inputs(case, seed)
    G, out = case["heads"] // case["kv_heads"], []
    at = 0
    for p, c, ks, vs in zip(past, new, k, v):
        ks, vs = _held(ks, case["bits"]), _held(vs, case["bits"])
        for i0 in range(0, c, 256):  # blocks of queries
            i1 = min(c, i0 + 256)
            e = p + i1
            y = []
            for h in range(case["heads"]):
                s = (q[at + i0: at + i1, h].double() @ ks[:e, h // G].T) * case["size"] ** -0.5
                s += torch.triu(torch.full_like(s, -math.inf), p + i0 + 1)
                y.append(torch.exp(s - torch.logsumexp(s, 1, keepdim=True)) @ vs[:e, h // G])
            out.append(torch.stack(y, 1))
        at += c
    return torch.cat(out)


def _exact_store(case, seed):
    past, new, old, k, v = _store_inputs(case, seed)
    cut = np.cumsum([0] + list(new))
    return tuple(_held(torch.cat([y for s in range(case["n"]) for y in (o[s], x[:, cut[s]: cut[s + 1]])], 1), case["bits"])
                 for o, x in zip(old, (k, v)))


def _exact_reorder(case, seed):
    old, k, v, parents = _reorder_inputs(case, seed)
    return tuple(_held(torch.cat([y for i, b in enumerate(parents) for y in (o[b], x[:, i: i + 1])], 1), case["bits"])
                 for o, x in zip(old, (k, v)))


def _exact_beam(case, seed):
    logits, scores, suppress = _beam_inputs(case, seed)
    W, V, n = case["width"], case["vocab"], case["best"]
    scores = scores.double().cpu().numpy()
    parents, tokens, out = [], [], []
    for g in range(case["groups"]):
        x = logits[g * W: (g + 1) * W].double().cpu().numpy()
        x[:, suppress] = -np.inf
        top = x.max(1, keepdims=True)
        x = (scores[g * W: (g + 1) * W, None] + (x - top - np.log(np.exp(x - top).sum(1, keepdims=True)))).ravel()
        some = np.nonzero(x >= np.partition(x, len(x) - min(n, len(x)))[len(x) - min(n, len(x))])[0]
        some = some[np.lexsort((some, -x[some]))][:n]
        some = some[x[some] > -np.inf]
        gap = n - len(some)
        parents.append(np.concatenate([some // V, np.full(gap, -1)]))
        tokens.append(np.concatenate([some % V, np.full(gap, -1)]))
        out.append(np.concatenate([x[some], np.full(gap, -np.inf)]))
    return np.array(parents, np.int32), np.array(tokens, np.int32), np.array(out)
