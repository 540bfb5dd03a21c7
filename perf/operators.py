"""Operators of sampled decoding over a paged key/value cache.

A recogniser that decodes several candidates of one segment (temperature
fallback with best-of-n, drafts to verify, long prompts of previous text) needs
three things besides the greedy step: a cache whose sequences can share, copy
and give back pages, attention of one or many new tokens over such a cache,
and the choice of a token from its logits with temperature, top-k, top-p and
min-p. Each case is one of

* op "attend": the attention of `n` sequences' new tokens (1 .. `new` each)
  over `past` cached positions at most and themselves, causal;
* op "fork": a sequence of `past` positions becomes `n` candidates, whose
  keys and values of all layers are then copied out (as a program does that
  moves them to another cache);
* op "append": the keys and values of `n` sequences' new tokens, all layers,
  are written behind what they hold, and the sequences copied out;
* op "sample": `rows` rows of `vocab` logits, options per row, one given
  uniform random number per row.

Plain forms keep pages as [layer][page][position][head][size] tensors and a
list of pages per sequence.
"""
import math

import numpy as np
import torch

own = False


def listed():
    def attend(name, dtype, n, past, new, heads, kv_heads, size, page):
        return {"name": name, "op": "attend", "dtype": dtype, "n": n, "past": past, "new": new, "heads": heads,
                "kv_heads": kv_heads, "size": size, "page": page}

    def pages(name, op, dtype, n, past, new, layers, kv_heads, size, page):
        return {"name": name, "op": op, "dtype": dtype, "n": n, "past": past, "new": new, "layers": layers,
                "kv_heads": kv_heads, "size": size, "page": page}

    def sample(name, dtype, rows, vocab, mix):
        return {"name": name, "op": "sample", "dtype": dtype, "rows": rows, "vocab": vocab, "mix": mix}

    return [
        # one step of one utterance on the smallest fp32 model: latency
        attend("attend-f32-step-1", "f32", 1, 37, 1, 6, 6, 64, 64),
        # one step of a full batch of the largest model, ragged
        attend("attend-step-32", "bf16", 32, 447, 1, 20, 20, 64, 64),
        # few rows over long contexts, grouped heads: the cache's bytes
        attend("attend-long-4", "bf16", 4, 60001, 1, 32, 8, 128, 128),
        # five drafted tokens per sequence to verify in one pass
        attend("attend-draft-16", "bf16", 16, 4001, 5, 16, 4, 64, 32),
        # ragged prompts of previous text run through at once
        attend("attend-prompts-9", "bf16", 9, 701, 513, 20, 20, 64, 64),
        # a long document's next chunk: the matrix cores
        attend("attend-fill-4096", "bf16", 1, 4097, 4096, 32, 8, 128, 64),
        # the fp32 model's prompts
        attend("attend-f32-prompts-16", "f32", 16, 40, 223, 8, 8, 64, 64),
        # best of five after a prompt of previous text, every layer of the largest model
        pages("fork-5", "fork", "bf16", 5, 229, 0, 32, 20, 64, 64),
        # prompts written behind earlier text, a small model's layers
        pages("append-16", "append", "bf16", 16, 101, 224, 12, 12, 64, 32),
        # one utterance's next token
        sample("sample-1", "f32", 1, 51865, "nucleus"),
        # a batch of users, each with options of its own
        sample("sample-32", "f32", 32, 51866, "all"),
        # many candidates over a wide vocabulary
        sample("sample-384", "bf16", 384, 151937, "all"),
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "fork", "append", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "sample":
        vocab = _log(rng, 33, 152000)
        return {"op": op, "dtype": dtype, "rows": _log(rng, 1, max(1, min(512, 20000000 // vocab))), "vocab": vocab,
                "mix": rng.choice(["nucleus", "top_k", "all"])}
    page = rng.choice([32, 64, 128])
    size = rng.choice([64, 64, 128])
    kv = rng.choice([1, 2, 4, 5, 8, 12, 16, 20])
    if op != "attend":
        layers = rng.choice([1, 4, 6, 12, 24, 32])
        n = _log(rng, 1, 16)
        top = max(2, 400000000 // (layers * kv * size * n * 4))  # positions per sequence
        return {"op": op, "dtype": dtype, "n": n, "past": _log(rng, 1, min(2000, top)),
                "new": _log(rng, 1, min(1000, top)) if op == "append" else 0, "layers": layers, "kv_heads": kv,
                "size": size, "page": page}
    group = rng.choice([1, 1, 2, 4, 5, 8])
    while group * kv > 40:
        group = rng.choice([1, 2])
    kind = rng.choice(["step", "step", "draft", "prompts"])
    new = {"step": 1, "draft": rng.randint(2, 8), "prompts": _log(rng, 9, 1500)}[kind]
    n = _log(rng, 1, {"step": 64, "draft": 32, "prompts": 16}[kind])
    cells = 200000000 if dtype == "bf16" else 60000000  # scores of one pass, and the cached numbers
    past = min(60000, max(1, cells // (n * new * kv * group)), max(1, cells // (n * kv * size)))
    return {"op": op, "dtype": dtype, "n": n, "past": _log(rng, 1, past), "new": new, "heads": kv * group,
            "kv_heads": kv, "size": size, "page": page}


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[case["dtype"]]


def _lengths(case):
    """Cached positions and new tokens of every sequence, the same for every
    seed: the first has the case's, the others a ragged share of them."""
    n, past, new = case["n"], case["past"], case["new"]
    r = np.random.RandomState(n * 1009 + past)
    p = [past] + [int(x) for x in r.randint(past // 16, past + 1, n - 1)]
    c = [new] + [int(x) for x in r.randint((new + 3) // 4, new + 1, n - 1)]
    return p, c


def _rows(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _attend_inputs(case, seed):
    past, new = _lengths(case)
    g, t = _generator(seed), _dtype(case)
    kv, size = case["kv_heads"], case["size"]
    k = [_rows(g, (p + c, kv, size), t) for p, c in zip(past, new)]
    v = [_rows(g, (p + c, kv, size), t) for p, c in zip(past, new)]
    q = _rows(g, (sum(new), case["heads"], size), t) * 1.5
    return past, new, q, k, v


def _pages_inputs(case, seed):
    g, t = _generator(seed), _dtype(case)
    shape = (case["kv_heads"], case["size"])
    if case["op"] == "fork":
        past, new = [case["past"]], [0]
    else:
        past, new = _lengths(case)
    old = [[_rows(g, (case["layers"], p, *shape), t) for p in past] for _ in range(2)]
    k, v = (_rows(g, (case["layers"], sum(new), *shape), t) for _ in range(2))
    return past, new, old, k, v


def _sample_inputs(case, seed):
    g = _generator(seed)
    r = np.random.RandomState(seed % 2**31)
    rows, V = case["rows"], case["vocab"]
    logits = torch.randn((rows, V), generator=g, device="cuda") * 2.5
    best = torch.randint(0, V, (rows, 5), generator=g, device="cuda")
    logits.scatter_add_(1, best, torch.rand((rows, 5), generator=g, device="cuda") * 14)
    # a range of ids ruled out by the program in every third row (timestamps before the last one)
    logits[::3, V - V // 34:] = -math.inf
    u = torch.rand(rows, generator=g, device="cuda")
    mix = case["mix"]
    opt = {"temperature": r.choice([0.2, 0.4, 0.6, 0.8, 1.0], rows), "top_k": np.zeros(rows, np.int32),
           "top_p": np.ones(rows), "min_p": np.zeros(rows)}
    if mix in ("nucleus", "all"):
        opt["top_p"] = r.choice([0.5, 0.9, 0.95, 1.0] if mix == "all" else [0.9, 0.95], rows)
    if mix in ("top_k", "all"):
        opt["top_k"] = r.choice([0, 1, 5, 40, 200, 1000] if mix == "all" else [5, 40, 200], rows)
    if mix == "all":
        opt["min_p"] = r.choice([0.0, 0.0, 0.02, 0.1], rows)
        opt["temperature"] = r.choice([0.0, 0.2, 0.4, 0.6, 0.8, 1.0, 1.3], rows)
    opt = {k: np.ascontiguousarray(x, np.int32 if k == "top_k" else np.float32) for k, x in opt.items()}
    suppress = np.unique(r.randint(0, V, min(88, V // 8))).astype(np.int32)  # never chosen, as set once for a model
    return logits.to(_dtype(case)), u, opt, suppress


# ------------------------------------------------------------------ preparation

def _cache(case, layers, kv, lens, heads=None):
    """The framework's cache, holding what lens says at most."""
    from paper_2507_01021_amd import binding
    P = case["page"]
    c = binding.Cache(dtype=binding.DTYPE_F32 if case["dtype"] == "f32" else binding.DTYPE_BF16, n_layer=layers,
                      n_head=heads or kv, n_kv_head=kv, head_size=case["size"], page_size=P,
                      n_pages=sum(-(-x // P) for x in lens) + 1, max_seqs=len(lens), max_positions=max(lens),
                      max_tokens=sum(lens))
    c.set_stream(torch.cuda.current_stream().cuda_stream)
    return c


def _fill(pages, lists, free, P, rows, lens):
    """Plain form: rows[s] [layer][position][...] into new pages of sequence s."""
    for s, n in enumerate(lens):
        lists[s] = [free.pop() for _ in range(-(-n // P))]
        _put(pages, lists[s], P, 0, rows[s])


def _put(pages, plist, P, first, rows):
    n = rows.shape[1]
    at = torch.arange(first, first + n, device="cuda")
    where = torch.tensor(plist, dtype=torch.long, device="cuda")[at // P]
    pages[:, where, at % P] = rows


def prepare(case, seed):
    op = case["op"]
    st = {"case": case}
    if op == "sample":
        st["logits"], st["u"], opt, suppress = _sample_inputs(case, seed)
        rows, V = case["rows"], case["vocab"]
        if own:
            from paper_2507_01021_amd import binding
            s = binding.Sampler(V, rows)
            s.set_stream(torch.cuda.current_stream().cuda_stream)
            s.options(suppress=suppress, **opt)
            st["sampler"] = s
            st["dt"] = binding.DTYPE_F32 if case["dtype"] == "f32" else binding.DTYPE_BF16
            st["tok"] = torch.empty(rows, dtype=torch.int32, device="cuda")
            st["lp"] = torch.empty(rows, dtype=torch.float32, device="cuda")
        else:
            st["opt"] = {k: torch.from_numpy(x).cuda() for k, x in opt.items()}
            st["suppress"] = torch.from_numpy(suppress.astype(np.int64)).cuda()
        return st
    P, kv, size, t = case["page"], case["kv_heads"], case["size"], _dtype(case)
    if op == "attend":
        past, new, q, k, v = _attend_inputs(case, seed)
        n, lens = len(past), [p + c for p, c in zip(past, new)]
        st["q"], st["new"], st["past"] = q, new, past
        if own:
            c = _cache(case, 1, kv, lens, case["heads"])
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
            lists, free = [None] * n, list(range(sum(-(-x // P) for x in lens)))
            order = np.random.RandomState(seed % 2**31).permutation(len(free))
            free = [int(x) for x in order]
            keep = list(free)
            st["k"], st["v"] = (torch.zeros((1, len(free), P, kv, size), dtype=t, device="cuda") for _ in range(2))
            for pages, rows in ((st["k"], k), (st["v"], v)):
                free = list(keep)
                _fill(pages, lists, free, P, [r[None] for r in rows], lens)
            st["pages"] = [torch.tensor(x, dtype=torch.long, device="cuda") for x in lists]
        return st
    past, new, old, k, v = _pages_inputs(case, seed)
    L, n = case["layers"], case["n"]
    ends = [case["past"]] * (n + 1) if op == "fork" else [p + c for p, c in zip(past, new)]
    total = n * case["past"] if op == "fork" else sum(ends)
    st["past"], st["new"], st["ends"], st["nk"], st["nv"] = past, new, ends, k, v
    st["k_out"], st["v_out"] = (torch.empty((L, total, kv, size), dtype=t, device="cuda") for _ in range(2))
    if own:
        c = _cache(case, L, kv, ends)
        some = [s for s in range(len(past)) if past[s]]
        if some:
            kk, vv = (torch.cat([x[s] for s in some], 1) for x in old)
            c.extend(some, [past[s] for s in some])
            c.append(-1, kk.data_ptr(), vv.data_ptr())
            torch.cuda.synchronize()
        st["cache"] = c
    else:
        count = sum(-(-x // P) for x in ends) + 1
        st["k"], st["v"] = (torch.zeros((L, count, P, kv, size), dtype=t, device="cuda") for _ in range(2))
        for pages, rows in ((st["k"], old[0]), (st["v"], old[1])):
            st["lists"], st["free"] = [[] for _ in ends], list(range(count - 1, -1, -1))
            _fill(pages, st["lists"], st["free"], P, rows, past)
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    case = st["case"]
    op = case["op"]
    if op == "sample":
        return _sample_own(st) if own else _sample_plain(st)
    if op == "attend":
        if own:
            st["cache"].attend(0, st["q"].data_ptr(), st["out"].data_ptr())
            return st["out"]
        return _attend_plain(st)
    n = case["n"]
    if op == "fork":
        copies = list(range(1, n + 1))
        if own:
            c = st["cache"]
            c.truncate(copies, [0] * n)
            c.fork(0, copies)
            c.read(-1, copies, st["k_out"].data_ptr(), st["v_out"].data_ptr())
            return st["k_out"], st["v_out"]
        return _fork_plain(st, copies)
    seqs = list(range(n))
    if own:
        c = st["cache"]
        c.truncate(seqs, st["past"])
        c.extend(seqs, st["new"])
        c.append(-1, st["nk"].data_ptr(), st["nv"].data_ptr())
        c.read(-1, seqs, st["k_out"].data_ptr(), st["v_out"].data_ptr())
        return st["k_out"], st["v_out"]
    return _append_plain(st)


def _attend_plain(st):
    case, q = st["case"], st["q"]
    H, kv, D, P = case["heads"], case["kv_heads"], case["size"], case["page"]
    G = H // kv
    out = torch.empty_like(q)
    r = 0
    for s, (p, c) in enumerate(zip(st["past"], st["new"])):
        k, v = (x[0, st["pages"][s]].reshape(-1, kv, D)[: p + c].float() for x in (st["k"], st["v"]))
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


def _gather(st, seqs, out_k, out_v):
    case, at = st["case"], 0
    P = case["page"]
    for s in seqs:
        n = st["ends"][s]
        where = torch.tensor(st["lists"][s], dtype=torch.long, device="cuda")
        for pages, out in ((st["k"], out_k), (st["v"], out_v)):
            out[:, at: at + n] = pages[:, where].flatten(1, 2)[:, :n]
        at += n
    return out_k, out_v


def _fork_plain(st, copies):
    P, n = st["case"]["page"], st["case"]["past"]
    full = n // P
    for s in copies:  # pages of their own go back, whole pages of the source are shared
        st["free"] += st["lists"][s][full:]
        st["lists"][s] = list(st["lists"][0][:full])
        if n % P:
            new = st["free"].pop()
            for pages in (st["k"], st["v"]):
                pages[:, new] = pages[:, st["lists"][0][full]]
            st["lists"][s].append(new)
    return _gather(st, copies, st["k_out"], st["v_out"])


def _append_plain(st):
    P, r = st["case"]["page"], 0
    for s, (p, c) in enumerate(zip(st["past"], st["new"])):
        keep = -(-p // P)
        st["free"] += st["lists"][s][keep:]
        st["lists"][s] = st["lists"][s][:keep] + [st["free"].pop() for _ in range(-(-(p + c) // P) - keep)]
        for pages, rows in ((st["k"], st["nk"]), (st["v"], st["nv"])):
            _put(pages, st["lists"][s], P, p, rows[:, r: r + c])
        r += c
    return _gather(st, range(len(st["past"])), st["k_out"], st["v_out"])


def _sample_own(st):
    x = st["logits"]
    st["sampler"].run(x.data_ptr(), st["dt"], x.shape[0], st["u"].data_ptr(), st["tok"].data_ptr(), st["lp"].data_ptr())
    return st["tok"], st["lp"]


def _sample_plain(st):
    """Temperature, then the top_k largest (lowest ids among equals), then the
    smallest prefix of them that holds top_p of their probability, then those
    of at least min_p times the largest's probability; the first id, in the
    order of ids, at which the kept probability passes u times its total."""
    o, V = st["opt"], st["case"]["vocab"]
    l = st["logits"].float().clone()
    l[:, st["suppress"]] = -math.inf
    top = l.amax(1, keepdim=True)
    d = l.double() - top.double()
    t = o["temperature"].double()[:, None]
    w = torch.exp(d / torch.where(t > 0, t, torch.ones_like(t)))
    order = torch.sort(l, dim=1, descending=True, stable=True).indices
    sw = torch.gather(w, 1, order)
    rank = torch.arange(V, device="cuda")[None]
    k = o["top_k"].long()[:, None]
    keep = rank < torch.where(k > 0, k, torch.full_like(k, V))
    keep &= (t > 0) | (rank < 1)
    sw = sw * keep
    cum = sw.cumsum(1)
    keep &= (cum - sw < o["top_p"].double()[:, None] * cum[:, -1:]) | (rank < 1)
    keep &= sw >= o["min_p"].double()[:, None]
    kept = torch.zeros_like(w).scatter_(1, order, sw * keep)
    cum = kept.cumsum(1)
    tok = (cum <= st["u"].double()[:, None] * cum[:, -1:]).sum(1)
    last = (kept > 0).long().mul(rank).amax(1)
    tok = torch.minimum(tok, last)
    lse = torch.exp(d).sum(1).log()
    lp = torch.gather(d, 1, tok[:, None])[:, 0] - lse
    return tok.int(), lp.float()


# ------------------------------------------------------------------ work and exact results

def work(case):
    op = case["op"]
    b = 4 if case["dtype"] == "f32" else 2
    if op == "sample":
        rows, V = case["rows"], case["vocab"]
        return {"bytes": rows * (V * b + 28), "flops": 10 * rows * V}
    kv, D = case["kv_heads"], case["size"]
    if op == "fork":
        one = 2 * case["layers"] * case["past"] * kv * D * b
        return {"bytes": one * (1 + case["n"]), "flops": 0}
    past, new = _lengths(case)
    if op == "append":  # what was there is read and copied out; new rows are read, written and copied out
        return {"bytes": 2 * case["layers"] * (2 * sum(past) + 3 * sum(new)) * kv * D * b, "flops": 0}
    H = case["heads"]
    return {"bytes": b * D * (2 * kv * (sum(past) + sum(new)) + 2 * H * sum(new)),
            "flops": sum(4 * H * D * c * (p + (c + 1) / 2) for p, c in zip(past, new))}


def exact(case, seed):
    op = case["op"]
    if op == "sample":
        return _sample_exact(case, seed)
    if op == "attend":
        past, new, q, k, v = _attend_inputs(case, seed)
        G, out = case["heads"] // case["kv_heads"], []
        at = 0
        for p, c, ks, vs in zip(past, new, k, v):
            for i0 in range(0, c, 256):  # blocks of queries, all heads of a block at once
                i1 = min(c, i0 + 256)
                e = p + i1
                qd = q[at + i0: at + i1].double()
                kd = ks[:e].double().repeat_interleave(G, 1)
                vd = vs[:e].double().repeat_interleave(G, 1)
                y = []
                for h in range(case["heads"]):
                    s = (qd[:, h] @ kd[:, h].T) * case["size"] ** -0.5
                    s += torch.triu(torch.full_like(s, -math.inf), p + i0 + 1)
                    y.append(torch.exp(s - torch.logsumexp(s, 1, keepdim=True)) @ vd[:, h])
                out.append(torch.stack(y, 1))
            at += c
        return torch.cat(out)
    past, new, old, k, v = _pages_inputs(case, seed)
    if op == "fork":
        return tuple(torch.cat([x[0]] * case["n"], 1).double() for x in old)
    cut = np.cumsum([0] + list(new))
    return tuple(torch.cat([y for s in range(case["n"]) for y in (o[s], x[:, cut[s]: cut[s + 1]])], 1).double()
                 for o, x in zip(old, (k, v)))


def _sample_exact(case, seed):
    logits, u, opt, suppress = _sample_inputs(case, seed)
    rows = logits.double().cpu().numpy()
    rows[:, suppress] = -np.inf
    u = u.double().cpu().numpy()
    toks, lps = [], []
    for i, l in enumerate(rows):
        t, k, tp, mp = (float(opt[x][i]) for x in ("temperature", "top_k", "top_p", "min_p"))
        m = l.max()
        ids = np.argsort(-l, kind="stable")
        ids = ids[np.isfinite(l[ids])]
        if t == 0:
            tok = int(ids[0])
        else:
            if k:
                ids = ids[: int(k)]
            p = np.exp((l[ids] - m) / t)
            p /= p.sum()
            before = np.concatenate([[0.0], np.cumsum(p)[:-1]])
            n = max(1, int(np.sum(before < tp)))
            n = min(n, int(np.sum(p >= mp * p[0])))
            kept = np.sort(ids[:n])
            c = np.cumsum(np.exp((l[kept] - m) / t))
            tok = int(kept[min(int(np.searchsorted(c, u[i] * c[-1], side="right")), n - 1)])
        toks.append(tok)
        lps.append(l[tok] - m - np.log(np.exp(l - m).sum()))
    return np.array(toks, np.int32), np.array(lps)
