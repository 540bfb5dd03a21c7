"""The sampler on the GPU against float64 NumPy: tokens equal, log-probabilities
within rounding."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2507_01021_amd import binding

pytestmark = pytest.mark.gpu


def choose(l, u, t, k, p, mp):
    """Token and log-probability of one row of float64 logits (inadmissible: -inf)."""
    l = np.where(np.isnan(l), -np.inf, l)
    m = l.max()
    if m == -np.inf:
        return -1, -np.inf
    with np.errstate(invalid="ignore"):
        d = np.where(l == m, 0.0, l - m)
    lse = np.log(np.exp(d).sum())
    ids = np.argsort(-l, kind="stable")
    ids = ids[l[ids] > -np.inf]
    if t == 0:
        return int(ids[0]), -lse
    if k:
        ids = ids[:k]
    w = np.exp(d[ids] / t)
    cum = np.cumsum(w)
    n = max(1, int(np.sum(cum - w < p * cum[-1]))) if p < 1 else len(ids)
    n = max(1, min(n, int(np.sum(w >= mp))))
    kept = np.sort(ids[:n])
    c = np.cumsum(np.exp(d[kept] / t))
    u = 0.0 if not u > 0 else u
    tok = int(kept[min(int(np.searchsorted(c, u * c[-1], side="right")), n - 1)])
    return tok, d[tok] - lse


def run(logits, u, opt, suppress=(), check=True, stride=0, sampler=None):
    rows, V = u.size, logits.shape[1]
    dt = binding.DTYPE_F32 if logits.dtype == torch.float32 else binding.DTYPE_BF16
    s = sampler or binding.Sampler(V, rows)
    s.options(suppress=suppress, n_rows=rows, **opt)
    ud = torch.from_numpy(u.astype(np.float32)).cuda()
    tok = torch.full((rows + 1,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((rows + 1,), -7.0, dtype=torch.float32, device="cuda")
    torch.cuda.synchronize()
    s.run(logits.data_ptr(), dt, rows, ud.data_ptr(), tok.data_ptr(), lp.data_ptr(), stride)
    torch.cuda.synchronize()
    assert tok[rows] == -7 and lp[rows] == -7
    tok2 = torch.empty_like(tok)
    s.run(logits.data_ptr(), dt, rows, ud.data_ptr(), tok2.data_ptr(), 0, stride)  # without log-probabilities
    torch.cuda.synchronize()
    assert torch.equal(tok[:rows], tok2[:rows])
    if not check:
        return tok[:rows].cpu().numpy(), lp[:rows].cpu().numpy()
    x = logits.double().cpu().numpy().copy()
    x[:, list(suppress)] = -np.inf
    uf = u.astype(np.float32).astype(np.float64)
    one = lambda a, i: np.asarray(a)[i] if np.ndim(a) else a
    for i in range(rows):
        o = [float(np.float32(one(opt.get(n, dflt), i))) for n, dflt in
             (("temperature", 1.0), ("top_p", 1.0), ("min_p", 0.0))]
        t, lpr = choose(x[i], uf[i], o[0], int(one(opt.get("top_k", 0), i)), o[1], o[2])
        assert int(tok[i]) == t, (i, int(tok[i]), t, o, one(opt.get("top_k", 0), i), u[i])
        got = float(lp[i])
        if t < 0:
            assert got == -np.inf
        else:
            # rounded to fp32 once (2^-24 of it); the logarithm of a sum whose terms are fp32
            # exponentials (relative error 2^-23 and 2^-24 of the argument, at most 100 where they count)
            assert abs(got - lpr) <= 2.0 ** -24 * abs(lpr) + 2.0 ** -22 + 100 * 2.0 ** -24, (i, got, lpr)
    return tok[:rows].cpu().numpy(), lp[:rows].cpu().numpy()


def logits_like_a_model(rows, V, seed, dtype=torch.float32, peak=14.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(rows, V, generator=g, device="cuda") * 2.5
    at = torch.randint(0, V, (rows, 5), generator=g, device="cuda")
    x.scatter_add_(1, at, torch.rand(rows, 5, generator=g, device="cuda") * peak)
    return x.to(dtype)


VOCABS = [1, 2, 33, 64, 1000, 51865, 51866, 131077]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", VOCABS)
def test_options_per_row(V, dtype):
    rows = 40
    r = np.random.RandomState(V)
    opt = {"temperature": r.choice([0.0, 0.05, 0.2, 0.7, 1.0, 1.5, 30.0], rows), "top_k": r.choice([0, 1, 2, 5, 40, 200, 10**6], rows),
           "top_p": r.choice([1.0, 0.99, 0.9, 0.5, 0.01], rows), "min_p": r.choice([0.0, 0.0, 0.02, 0.3, 1.0], rows)}
    sup = np.unique(r.randint(0, V, min(50, V // 3)))
    run(logits_like_a_model(rows, V, V, dtype), r.rand(rows), opt, sup)


@pytest.mark.parametrize("V", [33, 51865])
@pytest.mark.parametrize("opt", [dict(), dict(top_k=17), dict(top_p=0.9), dict(min_p=0.05),
                                 dict(top_k=50, top_p=0.8, min_p=0.01), dict(temperature=0.0), dict(temperature=8.0, top_p=0.97)])
def test_one_row(V, opt):
    r = np.random.RandomState(1)
    x = logits_like_a_model(8, V, 3)
    for i in range(8):
        run(x[i: i + 1], r.rand(1), opt)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [64, 30000])
def test_equal_logits_keep_the_lowest_ids(V, dtype):
    rows = 12
    x = torch.zeros(rows, V, dtype=dtype, device="cuda")
    x[1::2] = -0.0
    x[3::4, V // 2:] = 0.0
    u = np.linspace(0, 0.999, rows)
    tok, _ = run(x, u, dict(top_k=7))
    assert tok.max() < 7
    tok, _ = run(x, u, dict(top_p=0.5))
    assert tok.max() < V // 2
    run(x, u, dict(top_k=V - 1, top_p=0.25, min_p=1.0))
    # few distinct values
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    x = torch.randint(0, 4, (rows, V), generator=g, device="cuda").to(dtype)
    for k in (1, 10, V // 4, V // 2, V - 1, V):
        run(x, u, dict(top_k=k, top_p=0.7))


def test_inadmissible_logits():
    V, inf, nan = 5000, float("inf"), float("nan")
    x = logits_like_a_model(10, V, 5)
    x[0] = -inf
    x[1] = nan
    x[2] = -inf
    x[2, 4321] = -3e38
    x[3, 7], x[3, 99] = inf, inf
    x[4, ::2] = nan
    x[5, :4999] = -inf
    x[6, 17] = nan
    x[7] = torch.finfo(torch.float32).min
    x[8, ::3] = torch.finfo(torch.float32).min
    x[9, 5] = 3.4e38
    u = np.random.RandomState(2).rand(10)
    for opt in (dict(), dict(temperature=0.0), dict(top_k=3), dict(top_p=0.9), dict(min_p=0.5), dict(top_k=4999, top_p=0.3)):
        run(x, u, opt)
        run(x, u, opt, suppress=[4321, 7])


def test_ends_of_the_uniform_numbers():
    x = logits_like_a_model(6, 51866, 8)
    u = np.array([0.0, 1.0 - 2.0 ** -24, 1.0, -1.0, 5.0, float("nan")])
    for opt in (dict(), dict(top_k=3), dict(top_p=0.5)):
        a, _ = run(x, u, opt)
    few, _ = run(x, u, dict(top_k=3))
    ids = [np.sort(np.argsort(-x[i].cpu().numpy(), kind="stable")[:3]) for i in range(6)]
    assert [few[i] for i in (0, 3, 5)] == [ids[i][0] for i in (0, 3, 5)]
    assert [few[i] for i in (1, 2, 4)] == [ids[i][2] for i in (1, 2, 4)]


def test_extreme_temperatures():
    x = logits_like_a_model(4, 1000, 4) * 1e3
    u = np.array([0.1, 0.5, 0.9, 0.99])
    for t in (1e-30, 1e-3, 1e4, 3e38):
        run(x, u, dict(temperature=t))
        run(x, u, dict(temperature=t, top_p=0.6))


def test_a_row_is_chosen_alike_in_any_batch_and_type():
    """bf16 logits and the same numbers in fp32, alone and among others."""
    V = 20011
    x = logits_like_a_model(70, V, 6, torch.bfloat16)
    u = np.random.RandomState(0).rand(70)
    opt = dict(temperature=0.9, top_p=0.95)
    a, la = run(x, u, opt, check=False)
    b, lb = run(x.float(), u, opt, check=False)
    assert (a == b).all() and (la == lb).all()
    for i in (0, 33, 69):
        c, lc = run(x[i: i + 1], u[i: i + 1], opt, check=False)
        assert c[0] == a[i] and lc[0] == la[i]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_and_unaligned_rows(dtype):
    V, ld = 4099, 4200 + 1
    base = torch.full((9 * ld + 3,), 50.0, dtype=dtype, device="cuda")
    rows = base[1: 1 + 9 * ld].view(9, ld)[:, :V]
    rows.copy_(logits_like_a_model(9, V, 2))
    run(rows, np.random.RandomState(3).rand(9), dict(top_p=0.9, top_k=100), stride=ld)


def test_frequencies_follow_the_probabilities():
    """Evenly spaced uniform numbers: every id is chosen within one of its share."""
    V, n = 50, 4096
    x = logits_like_a_model(1, V, 11, peak=2.0)
    tok, _ = run(x.expand(n, V).contiguous(), (np.arange(n) + 0.5) / n, dict(temperature=1.3), check=False)
    p = np.exp((x[0].double().cpu().numpy() - float(x.max())) / np.float64(np.float32(1.3)))
    share = n * p / p.sum()
    assert (np.abs(np.bincount(tok, minlength=V) - share) <= 1 + 1e-3).all()
    assert (np.diff(tok) >= 0).all()


def test_recorded_choice():
    """A recorded run takes the logits, numbers and options of its replay."""
    V, rows = 30011, 16
    s = binding.Sampler(V, rows)
    st = torch.cuda.Stream()
    s.set_stream(st.cuda_stream)
    x = torch.zeros(rows, V, device="cuda")
    u = torch.zeros(rows, device="cuda")
    tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
    lp = torch.zeros(rows, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        s.run(x.data_ptr(), 0, rows, u.data_ptr(), tok.data_ptr(), lp.data_ptr())
        with pytest.raises(binding.WhisperError) as e:
            s.options(temperature=0.3)
        assert e.value.status == binding.E_STATE
    r = np.random.RandomState(7)
    for i in range(4):
        opt = dict(temperature=0.5 + i, top_p=[1.0, 0.9, 0.5, 0.99][i], top_k=[0, 20, 0, 5][i])
        s.options(**opt)
        x.copy_(logits_like_a_model(rows, V, 100 + i))
        un = r.rand(rows).astype(np.float32)
        u.copy_(torch.from_numpy(un))
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        want, wl = run(x, un, opt, check=True)
        assert (tok.cpu().numpy() == want).all() and (lp.cpu().numpy() == wl).all()


def test_more_rows_than_the_workspace_holds():
    V, rows = 257, 1300
    r = np.random.RandomState(12)
    run(logits_like_a_model(rows, V, 12), r.rand(rows), dict(temperature=r.choice([0.0, 0.7, 1.0], rows), top_k=r.choice([0, 9], rows),
                                                             top_p=r.choice([1.0, 0.8], rows)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_wide_nuclei_and_long_lists(dtype):
    """Filters that keep tens of thousands of ids: more than the list of a row
    holds, bins of thousands of equal logits, ids sorted by their logits."""
    V = 120001
    x = logits_like_a_model(8, V, 13, dtype, peak=1.0)
    x[1] = x[1].sort(descending=True).values
    x[2] = x[2].sort().values
    x[3] = (x[3].float() * 2).round().to(dtype) / 2
    x[4] = 0
    x[5, : V // 2] = 3
    u = np.random.RandomState(14).rand(8)
    for opt in (dict(top_p=0.999), dict(top_p=0.5), dict(top_k=50000), dict(top_k=100000, top_p=0.9), dict(top_k=40000, top_p=0.99, min_p=1e-4),
                dict(temperature=20.0, top_p=0.7), dict(temperature=0.3, top_k=60000), dict(top_p=0.9, min_p=0.5)):
        run(x, u, opt)


def test_other_stream():
    x = logits_like_a_model(4, 5000, 15)
    u = torch.rand(4, device="cuda")
    s = binding.Sampler(5000, 4)
    s.options(top_p=0.9)
    toks = []
    st = torch.cuda.Stream()
    for handle in (None, st.cuda_stream, None):
        s.set_stream(handle)
        torch.cuda.synchronize()
        t = torch.empty(4, dtype=torch.int32, device="cuda")
        s.run(x.data_ptr(), 0, 4, u.data_ptr(), t.data_ptr())
        torch.cuda.synchronize()
        toks.append(t.tolist())
    assert toks[0] == toks[1] == toks[2]


def test_suppress_lists_set_after_the_recording():
    """A recorded run takes the ids suppressed when it is replayed, whether or
    not there were any when it was recorded."""
    V, rows = 5003, 4
    s = binding.Sampler(V, rows)
    st = torch.cuda.Stream()
    s.set_stream(st.cuda_stream)
    x = logits_like_a_model(rows, V, 21)
    un = np.array([0.1, 0.4, 0.7, 0.95])
    u = torch.from_numpy(un.astype(np.float32)).cuda()
    tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
    lp = torch.zeros(rows, device="cuda")
    torch.cuda.synchronize()
    best = [int(i) for i in x.argmax(1)]
    for before in ((), best):
        s.options(top_p=0.9, suppress=before)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            s.run(x.data_ptr(), 0, rows, u.data_ptr(), tok.data_ptr(), lp.data_ptr())
        for sup in ((), best, (), range(2500, V), before):
            s.options(top_p=0.9, suppress=list(sup))
            with torch.cuda.stream(st):
                g.replay()
            torch.cuda.synchronize()
            want, wl = run(x, un, dict(top_p=0.9), suppress=list(sup))
            assert not set(tok.tolist()) & set(sup)
            assert (tok.cpu().numpy() == want).all() and (lp.cpu().numpy() == wl).all(), len(sup)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_temperatures_at_the_ends_of_the_range(dtype):
    """Logits as far apart as the type allows at the highest temperatures (their
    difference exceeds fp32, their weights do not vanish), and denormal ones at
    the lowest: the filters count every id that has a weight. (A log-probability
    below fp32's range, of a logit 6.6e38 below the largest, is rounded to -inf.)"""
    def check_ends(x, u, opt):
        tok, lp = run(x, u, opt, check=False)
        o = {n: float(np.float32(opt.get(n, d))) for n, d in (("temperature", 1.0), ("top_p", 1.0), ("min_p", 0.0))}
        for i, l in enumerate(x.double().cpu().numpy()):
            t, want = choose(l, float(np.float32(u[i])), o["temperature"], opt.get("top_k", 0), o["top_p"], o["min_p"])
            assert tok[i] == t, (i, int(tok[i]), t, opt)
            with np.errstate(over="ignore"):
                w = np.float32(want)
            # as in run(): rounded once, a sum of fp32 exponentials
            assert lp[i] == w or abs(float(lp[i]) - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -22 + 100 * 2.0 ** -24, (i, lp[i], want)

    V = 200
    g = torch.Generator(device="cuda")
    g.manual_seed(17)
    big = ((torch.rand(6, V, generator=g, device="cuda") * 2 - 1) * 3.3e38).to(dtype)
    big[0, ::2], big[0, 1::2] = 3.3e38, -3.3e38
    u = np.linspace(0.02, 0.98, 6)
    filters = (dict(), dict(top_k=150), dict(top_p=0.9), dict(top_k=180, top_p=0.97), dict(top_p=0.99, min_p=0.2))
    for t in (3.4e38, 1e38, 2e37):
        for f in filters:
            check_ends(big, u, dict(temperature=t, **f))
    tiny = (torch.randint(-400, 400, (6, V), generator=g, device="cuda").double() * 2.0 ** -133).float().to(dtype)
    for t in (200 * 2.0 ** -133, 20 * 2.0 ** -133, 2.0 ** -149):
        for f in filters:
            check_ends(tiny, u, dict(temperature=t, **f))
