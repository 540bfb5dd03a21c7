"""The paged cache on the GPU against plain float64: rows in and out, forks,
compaction, and causal attention of one token and of chunks over pages."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2507_01021_amd import binding

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, binding.DTYPE_F32), "bf16": (torch.bfloat16, binding.DTYPE_BF16)}


class Pair:
    """A cache beside the plain rows of its sequences."""

    def __init__(self, dtype, H, Hkv, D, P, max_seqs, max_positions, layers=1, n_pages=None, max_tokens=None, seed=0):
        self.t, code = DT[dtype]
        self.H, self.Hkv, self.D, self.layers = H, Hkv, D, layers
        n_pages = n_pages or max_seqs * (-(-max_positions // P))
        self.c = binding.Cache(code, layers, H, Hkv, D, P, n_pages, max_seqs, max_positions,
                               max_tokens or max_seqs * max_positions)
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        e = torch.empty(layers, 0, Hkv, D, dtype=self.t, device="cuda")
        self.k, self.v = ([e] * max_seqs for _ in range(2))

    def rows(self, n, heads=None):
        return torch.randn(self.layers, n, heads or self.Hkv, self.D, generator=self.g, device="cuda").to(self.t)

    def add(self, seqs, counts, k=None, v=None, one_by_one=False):
        n = sum(counts)
        k = self.rows(n) if k is None else k
        v = self.rows(n) if v is None else v
        self.c.extend(seqs, counts)
        if one_by_one:
            for l in range(self.layers):
                self.c.append(l, k[l].data_ptr(), v[l].data_ptr())
        else:
            self.c.append(-1, k.data_ptr(), v.data_ptr())
        at = 0
        for s, m in zip(seqs, counts):
            self.k[s] = torch.cat([self.k[s], k[:, at: at + m]], 1)
            self.v[s] = torch.cat([self.v[s], v[:, at: at + m]], 1)
            at += m
        torch.cuda.synchronize()

    def cut(self, seqs, lens):
        self.c.truncate(seqs, lens)
        for s, n in zip(seqs, lens):
            self.k[s], self.v[s] = self.k[s][:, :n], self.v[s][:, :n]

    def check_rows(self, seqs):
        n = sum(self.k[s].shape[1] for s in seqs)
        ko = torch.full((self.layers, n, self.Hkv, self.D), 7.0, dtype=self.t, device="cuda")
        vo = ko.clone()
        self.c.read(-1, seqs, ko.data_ptr(), vo.data_ptr())
        torch.cuda.synchronize()
        assert torch.equal(ko, torch.cat([self.k[s] for s in seqs], 1))
        assert torch.equal(vo, torch.cat([self.v[s] for s in seqs], 1))

    def attend(self, seqs, counts, layer=0, q=None, scale=None):
        n = sum(counts)
        q = self.rows(n, self.H)[0] if q is None else q
        out = torch.full((n + 1, self.H, self.D), 7.0, dtype=self.t, device="cuda")
        self.c.attend(layer, q.data_ptr(), out.data_ptr(), scale=scale)
        torch.cuda.synchronize()
        assert (out[n] == 7).all()  # the row behind the last token is left alone
        self.check(out[:n], q, seqs, counts, layer, scale)
        return out[:n]

    def check(self, out, q, seqs, counts, layer=0, scale=None):
        scale = self.D ** -0.5 if scale is None else scale
        G, at = self.H // self.Hkv, 0
        for s, m in zip(seqs, counts):
            k, v = (x[s][layer].double().repeat_interleave(G, 1).transpose(0, 1) for x in (self.k, self.v))
            past = k.shape[1] - m
            for i0 in range(0, m, 512):
                i1 = min(m, i0 + 512)
                e = past + i1
                qs = q[at + i0: at + i1].double().transpose(0, 1)
                hidden = torch.arange(e, device="cuda")[None] > torch.arange(past + i0, past + i1, device="cuda")[:, None]
                sc = (torch.matmul(qs, k[:, :e].transpose(1, 2).contiguous()) * scale).masked_fill(hidden, -math.inf)
                w = torch.softmax(sc, -1)
                # a visible value may be infinite; hidden ones do not enter
                vz = torch.where(torch.isfinite(v[:, :e]), v[:, :e], torch.zeros_like(v[:, :e]))
                ref = torch.matmul(w, vz)
                mean = torch.matmul(w, vz.abs())
                # rounding: D products and sums of a score in fp32 (2^-24 each), relative error of a weight
                # twice that of the exponent's argument; sums over the positions in fp32; the hardware
                # exponential 2^-21; bf16: every weight and the output are rounded once (2^-8 each)
                es = (self.D + 4) * 2.0 ** -24 * scale * torch.matmul(qs.abs(), k[:, :e].abs().transpose(1, 2).contiguous()).amax()
                one = torch.finfo(self.t).eps / 2
                rel = 4 * es + 2.0 ** -20 + 2 * e * 2.0 ** -24 + (one if self.t == torch.bfloat16 else 0)
                tol = one * ref.abs() + rel * mean * (1 + one) + 1e-30
                err = (out[at + i0: at + i1].double().transpose(0, 1) - ref).abs()
                bad = ~(err <= tol)
                assert not bad.any(), (s, m, past, float((err / tol).nan_to_num(1e9).max()), bad.nonzero()[0].tolist())
            at += m


HEADS = [(6, 6, 64), (20, 20, 64), (8, 2, 64), (5, 1, 64), (32, 8, 128), (3, 3, 128), (24, 1, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,D", HEADS)
@pytest.mark.parametrize("P", [32, 128])
def test_rows_come_back(dtype, H, Hkv, D, P):
    p = Pair(dtype, H, Hkv, D, P, 5, 500, layers=3)
    p.add([0, 3, 1], [1, 131, 64])
    p.check_rows([0, 1, 3])
    p.add([1, 0, 2], [63, 31, 1], one_by_one=True)
    p.add([3], [1])
    p.check_rows([3, 2, 1, 0, 4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,D", HEADS)
@pytest.mark.parametrize("P", [32, 64, 128, 256])
def test_one_token_per_sequence(dtype, H, Hkv, D, P):
    p = Pair(dtype, H, Hkv, D, P, 7, 700, seed=P)
    p.add([0, 1, 2, 3, 4, 5], [31, 32, 33, 447, 127, 640])
    seqs = [5, 0, 1, 2, 3, 6, 4]  # 6: its first token
    for _ in range(3):
        p.add(seqs, [1] * 7)
        p.attend(seqs, [1] * 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,D", HEADS)
@pytest.mark.parametrize("P", [32, 64])
def test_chunks(dtype, H, Hkv, D, P):
    p = Pair(dtype, H, Hkv, D, P, 6, 900, seed=P + 1)
    p.add([0, 1, 2], [100, 5, 300])
    seqs, counts = [3, 0, 2, 1, 4, 5], [257, 1, 64, 0, 16, 200]
    p.add(seqs, counts)
    p.attend(seqs, counts)
    p.add([3, 1], [7, 333])
    p.attend([3, 1], [7, 333])


@pytest.mark.parametrize("dtype,H,Hkv,D,lens", [("bf16", 8, 2, 128, [20000, 1, 4097]), ("bf16", 20, 20, 64, [9000]),
                                                ("f32", 4, 1, 64, [12345, 700]), ("bf16", 1, 1, 64, [50000])])
def test_long_contexts_are_cut_and_joined(dtype, H, Hkv, D, lens):
    n = len(lens)
    p = Pair(dtype, H, Hkv, D, 128, n, max(lens) + 100)
    p.add(list(range(n)), lens)
    for counts in ([1] * n, [3] * n, [17] * n):
        p.add(list(range(n)), counts)
        p.attend(list(range(n)), counts)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_results_do_not_depend_on_pages(dtype):
    """Other pages, and a compaction: the same bits."""
    outs = []
    for mess in (False, True):
        p = Pair(dtype, 4, 2, 64, 32, 4, 600, n_pages=80, seed=3)
        if mess:
            p.c.extend([3, 2], [90, 40])
        k, v = (torch.randn(1, 500, 2, 64, generator=p.g, device="cuda").to(p.t) for _ in range(2))
        q = torch.randn(20, 4, 64, generator=p.g, device="cuda").to(p.t)
        p.add([0], [480], k[:, :480], v[:, :480])
        if mess:
            p.c.truncate([3, 2], [0, 0])
            p.c.compact()
        p.add([0], [20], k[:, 480:], v[:, 480:])
        outs.append(p.attend([0], [20], q=q))
        p.check_rows([0])
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("past", [1, 64, 229])
def test_forks_go_their_own_way(dtype, past):
    p = Pair(dtype, 4, 4, 64, 64, 6, 300, layers=2, seed=past)
    p.add([0], [past])
    p.c.fork(0, [1, 2, 5])
    for s in (1, 2, 5):
        p.k[s], p.v[s] = p.k[0], p.v[0]
    p.check_rows([0, 1, 2, 5])
    for step in range(3):
        p.add([5, 0, 1, 2], [1, 2, 1, 1])
        for l in (0, 1):
            p.attend([5, 0, 1, 2], [1, 2, 1, 1], layer=l)
    p.cut([1, 2], [past - 1, past + 1])  # drafted tokens taken back: shared pages stay whole
    p.add([1, 2, 0], [3, 1, 1])
    p.attend([1, 2, 0], [3, 1, 1], layer=1)
    p.check_rows([0, 1, 2, 5])
    p.cut([0], [0])
    p.c.compact()
    p.check_rows([1, 2, 5])
    p.add([1, 2, 5], [1, 1, 1])
    p.attend([1, 2, 5], [1, 1, 1])


@pytest.mark.parametrize("left_over", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_what_is_hidden_does_not_enter(dtype, D, left_over):
    """Infinities and NaN at later positions of the chunk, and left over in
    freed pages, reach no row that does not see them."""
    p = Pair(dtype, 4, 2, D, 32, 2, 600, n_pages=40)
    if left_over:
        bad = torch.full((1, 600, 2, D), math.nan, device="cuda").to(p.t)
        p.c.extend([1], [600])
        p.c.append(-1, bad.data_ptr(), bad.data_ptr())
        torch.cuda.synchronize()
        p.c.truncate([1], [0])
    for past, m in ((0, 1), (3, 1), (37, 9), (64, 300)):
        p.cut([0], [0])
        p.add([0], [past])
        k, v = p.rows(m), p.rows(m)
        for i, x in ((m - 1, math.inf), (m // 2 + 1, math.nan)):
            if 0 < i < m:
                v[0, i, :, 5] = x
        if m > 2:
            k[0, m - 1, 0] = math.nan
        p.add([0], [m], k, v)
        out = torch.empty(m, 4, D, dtype=p.t, device="cuda")
        q = p.rows(m, 4)[0]
        p.c.attend(0, q.data_ptr(), out.data_ptr())
        torch.cuda.synchronize()
        clean = min(i for i in (m - 1, m // 2 + 1) if i > 0) if m > 1 else m
        if m > 1:
            assert torch.isnan(out[m - 1, :2]).all()  # a visible NaN key
            assert not torch.isfinite(out[m // 2 + 1:, :, 5].float()).any()
        # the clean rows, against the plain rows cut there
        k0, v0 = p.k[0], p.v[0]
        p.k[0], p.v[0] = k0[:, : past + clean], v0[:, : past + clean]
        p.check(out[:clean], q, [0], [clean])
        p.k[0], p.v[0] = k0, v0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_unaligned_rows(dtype):
    """Rows cut out of a fused projection's output; keys and values at any address."""
    H, Hkv, D = 4, 2, 64
    p = Pair(dtype, H, Hkv, D, 64, 2, 400)
    n = 75
    fused = torch.randn(n, (H + 2 * Hkv) * D + 8, generator=p.g, device="cuda").to(p.t)
    ld = fused.stride(0)
    q, k, v = fused[:, : H * D], fused[:, H * D: (H + Hkv) * D], fused[:, (H + Hkv) * D: (H + 2 * Hkv) * D]
    p.c.extend([1], [n])
    p.c.append(0, k.data_ptr(), v.data_ptr(), ld, ld)
    out = torch.full((n, H * D + 16), 7.0, dtype=p.t, device="cuda")
    p.c.attend(0, q.data_ptr(), out.data_ptr(), ld, out.stride(0))
    torch.cuda.synchronize()
    assert (out[:, H * D:] == 7).all()
    p.k[1], p.v[1] = k.reshape(1, n, Hkv, D), v.reshape(1, n, Hkv, D)
    p.check(out[:, : H * D].reshape(n, H, D), q.reshape(n, H, D), [1], [n])
    # an odd address and odd strides
    odd = torch.randn(n * 401 + 1, generator=p.g, device="cuda").to(p.t)
    ko = odd[1:].view(n, 401)[:, 3: 3 + Hkv * D]
    vo = odd[1:].view(n, 401)[:, 200: 200 + Hkv * D]
    p.c.extend([0], [n])
    p.c.append(0, ko.data_ptr(), vo.data_ptr(), 401, 401)
    p.k[0], p.v[0] = ko.reshape(1, n, Hkv, D), vo.reshape(1, n, Hkv, D)
    back = torch.zeros(2, n * 301 + 1, dtype=p.t, device="cuda")
    kb, vb = (b[1:].view(n, 301) for b in back)
    p.c.read(0, [0], kb.data_ptr(), vb.data_ptr(), 301, 301)
    torch.cuda.synchronize()
    assert torch.equal(kb[:, : Hkv * D], ko) and torch.equal(vb[:, : Hkv * D], vo)
    assert not kb[:, Hkv * D:].any() and not back[:, 0].any()


def test_scale_and_large_scores():
    p = Pair("bf16", 2, 2, 64, 32, 1, 300)
    p.add([0], [200])
    p.add([0], [5])
    p.attend([0], [5], scale=3.0)  # nearly one-hot weights
    p.attend([0], [5], scale=1e-4)  # nearly equal ones


def test_other_stream():
    p = Pair("bf16", 4, 4, 64, 32, 2, 300)
    p.add([0], [100])
    st = torch.cuda.Stream()
    p.c.set_stream(st.cuda_stream)
    with torch.cuda.stream(st):
        p.add([0], [40])
        p.attend([0], [40])
    p.c.set_stream(None)
    p.add([0], [3])
    p.attend([0], [3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_recorded_step_serves_later_chunks(dtype):
    """append and attend in a graph, replayed for chunks of other lengths and
    sequences, with the program's own work between the replays."""
    n = 4
    p = Pair(dtype, 8, 4, 64, 32, 6, 3000, max_tokens=12000)
    p.add([0, 1, 2, 3, 4, 5], [100, 2500, 7, 1000, 31, 32])
    k, v = (torch.zeros(1, n, 4, 64, dtype=p.t, device="cuda") for _ in range(2))
    q = torch.zeros(n, 8, 64, dtype=p.t, device="cuda")
    out = torch.zeros(n, 8, 64, dtype=p.t, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    p.c.set_stream(st.cuda_stream)
    p.c.extend([0, 2, 4, 5], [1, 1, 1, 1])
    p.c.append(0, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    for s in (0, 2, 4, 5):
        p.k[s], p.v[s] = (torch.cat([x[s], torch.zeros_like(k[:, :1])], 1) for x in (p.k, p.v))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        p.c.append(0, k.data_ptr(), v.data_ptr())
        p.c.attend(0, q.data_ptr(), out.data_ptr())
        with pytest.raises(binding.WhisperError) as e:
            p.c.extend([0], [1])
        assert e.value.status == binding.E_STATE
    for seqs in ([0, 2, 4, 5], [1, 3, 0, 2], [1, 5, 4, 3]):
        p.c.extend(seqs, [1] * n)
        with torch.cuda.stream(st):
            for x in (k, v, q):
                x.copy_(torch.randn(x.shape, generator=p.g, device="cuda"))
            torch.cuda.synchronize()
            g.replay()
        torch.cuda.synchronize()
        for i, s in enumerate(seqs):
            p.k[s], p.v[s] = torch.cat([p.k[s], k[:, i: i + 1]], 1), torch.cat([p.v[s], v[:, i: i + 1]], 1)
        p.check(out, q, seqs, [1] * n)
        (torch.randn(64, 64, device="cuda") @ torch.randn(64, 64, device="cuda")).sum().item()


def test_state_errors():
    p = Pair("bf16", 2, 2, 64, 32, 2, 100)
    x = torch.zeros(200, 2, 64, dtype=torch.bfloat16, device="cuda").data_ptr()
    for f in (lambda: p.c.append(0, x, x), lambda: p.c.attend(0, x, x)):
        with pytest.raises(binding.WhisperError) as e:
            f()
        assert e.value.status == binding.E_STATE
    p.add([0], [40])
    p.c.truncate([0], [39])
    with pytest.raises(binding.WhisperError) as e:
        p.c.attend(0, x, x)
    assert e.value.status == binding.E_STATE
    p.k[0], p.v[0] = p.k[0][:, :39], p.v[0][:, :39]
    p.c.extend([0, 1], [0, 0])  # an empty chunk
    p.c.append(0, x, x)
    p.c.attend(0, x, x)
    p.check_rows([0])


def test_offsets_beyond_32_bits():
    """Pages behind the first 4 GiB of a cache's memory, in its last layer."""
    H, D, P, layers = 8, 128, 256, 32
    c = binding.Cache(binding.DTYPE_F32, layers, H, H, D, P, 100, 2, 90 * P, 90 * P)  # 67 MB a page
    c.extend([0], [80 * P])  # pages 0 .. 79, 5.4 GB
    n = 300
    k, v, q = (torch.randn(n, H, D, device="cuda") for _ in range(3))
    c.extend([1], [n])
    out = torch.empty_like(q)
    for layer in (0, layers - 1):
        c.append(layer, k.data_ptr(), v.data_ptr())
        c.attend(layer, q.data_ptr(), out.data_ptr())
        torch.cuda.synchronize()
        s = torch.matmul(q.double().transpose(0, 1), k.double().permute(1, 2, 0).contiguous()) * D ** -0.5
        s += torch.full((n, n), -math.inf, device="cuda").double().triu(1)
        ref = torch.matmul(torch.softmax(s, -1), v.double().transpose(0, 1).contiguous()).transpose(0, 1)
        # rounding as in Pair.check, with |q . k| D ** -0.5 below 64 and |v| below 6
        assert (out.double() - ref).abs().max() <= 6 * (4 * (D + 4) * 2.0 ** -24 * 64 + 2.0 ** -20 + 2 * n * 2.0 ** -24)
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    c.read(layers - 1, [1], kb.data_ptr(), vb.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(kb, k) and torch.equal(vb, v)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_in_place_of_queries(dtype):
    p = Pair(dtype, 8, 2, 64, 32, 3, 3000, seed=4)
    p.add([0, 1, 2], [2600, 70, 0])
    for counts in ([1, 5, 3], [40, 200, 1]):
        p.add([0, 1, 2], counts)
        q = p.rows(sum(counts), 8)[0]
        x = q.clone()
        p.c.attend(0, x.data_ptr(), x.data_ptr())
        torch.cuda.synchronize()
        p.check(x, q, [0, 1, 2], counts)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_minus_infinity_weigh_nothing(dtype, D):
    """Keys that make a score -inf, or the type's lowest value, over whole blocks
    in front of, between and behind the others."""
    low = torch.finfo(DT[dtype][0]).min
    for past, m in ((300, 1), (300, 5), (300, 200)):
        p = Pair(dtype, 4, 2, D, 64, 1, 600)
        k, v = p.rows(past + m), p.rows(past + m)
        q = p.rows(m, 4)[0]
        q[..., 0] = 1.0
        gone = torch.zeros(past + m, dtype=torch.bool, device="cuda")
        gone[:130] = True
        gone[190:256] = True
        gone[past + m // 2: past + m - 1: 2] = True
        for value in (-math.inf, low):
            kk = k.clone()
            kk[0, gone, :, 0] = value
            c = binding.Cache(DT[dtype][1], 1, 4, 2, D, 64, 20, 1, 600, 600)
            c.extend([0], [past])
            kp, vp = kk[:, :past].contiguous(), v[:, :past].contiguous()
            c.append(0, kp.data_ptr(), vp.data_ptr())
            torch.cuda.synchronize()
            c.extend([0], [m])
            kn, vn = kk[:, past:].contiguous(), v[:, past:].contiguous()
            c.append(0, kn.data_ptr(), vn.data_ptr())
            out = torch.empty_like(q)
            c.attend(0, q.data_ptr(), out.data_ptr())
            torch.cuda.synchronize()
            keep = ~gone
            for i in range(m):
                at = keep[: past + i + 1].nonzero()[:, 0]
                s = torch.einsum("hd,thd->ht", q[i].double().cpu(), k[0, at].double().cpu().repeat_interleave(2, 1)) * D ** -0.5
                w = torch.softmax(s, -1)
                x = v[0, at].double().cpu().repeat_interleave(2, 1)
                ref = torch.einsum("ht,thd->hd", w, x)
                mean = torch.einsum("ht,thd->hd", w, x.abs())
                one = torch.finfo(p.t).eps / 2
                # rounding as in Pair.check; |q| |k| D ** -0.5 summed over D stays below 64
                rel = 4 * (D + 4) * 2.0 ** -24 * 64 + 2.0 ** -20 + 2 * 600 * 2.0 ** -24 + (one if p.t == torch.bfloat16 else 0)
                err = (out[i].double().cpu() - ref).abs()
                assert (err <= one * ref.abs() + rel * mean * (1 + one)).all(), (past, m, value, i)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 7, 200])
def test_all_scores_the_lowest_value(dtype, D, m):
    """Equal scores weigh alike, also where they are the type's lowest value."""
    p = Pair(dtype, 4, 2, D, 64, 1, 600)
    k, v = p.rows(300 + m), p.rows(300 + m)
    k[..., 0] = torch.finfo(p.t).min
    q = p.rows(m, 4)[0]
    q[..., 0] = 1.0
    for at, n in ((0, 300), (300, m)):
        p.c.extend([0], [n])
        kn, vn = k[:, at:at + n].contiguous(), v[:, at:at + n].contiguous()
        p.c.append(0, kn.data_ptr(), vn.data_ptr())
        torch.cuda.synchronize()
    out = torch.empty_like(q)
    p.c.attend(0, q.data_ptr(), out.data_ptr())
    torch.cuda.synchronize()
    x = v[0].double().cpu().repeat_interleave(2, 1)
    one = torch.finfo(p.t).eps / 2
    for i in range(m):
        n = 301 + i
        ref, mean = x[:n].mean(0), x[:n].abs().mean(0)
        # weights of 1, summed over n positions in float32; the output is rounded
        err = (out[i].double().cpu() - ref).abs()
        assert (err <= one * ref.abs() + 2 * n * 2.0 ** -24 * mean * (1 + one)).all(), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_replay_without_a_chunk(dtype):
    """A truncate that ends the chunk also ends it for recorded launches: the
    freed pages, which another sequence holds now, and the outputs stay."""
    p = Pair(dtype, 4, 2, 64, 32, 2, 200)
    p.add([0], [70])
    k, v, q = p.rows(80), p.rows(80), p.rows(80, 4)[0]
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    p.c.set_stream(st.cuda_stream)
    p.c.extend([0], [40])
    p.c.append(0, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        p.c.append(0, k.data_ptr(), v.data_ptr())
        p.c.attend(0, q.data_ptr(), out.data_ptr())
        with pytest.raises(binding.WhisperError) as e:
            p.c.truncate([0], [70])
        assert e.value.status == binding.E_STATE
    p.c.set_stream(0)
    for _ in range(2):
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        p.k[0], p.v[0] = torch.cat([p.k[0][:, :70], k[:, :40]], 1), torch.cat([p.v[0][:, :70], v[:, :40]], 1)
        p.check(out, q, [0], [40])
        p.cut([0], [0])
        p.add([1], [70])  # from the freed pages
        p.cut([1], [69])
        before = out.clone()
        k.add_(1)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, before)
        p.check_rows([1])
        p.cut([1], [0])
        p.add([0], [70])
        p.c.extend([0], [40])
        torch.cuda.synchronize()


def recorded(p, st, *calls):
    """The calls in a graph on stream st, which the cache gets."""
    torch.cuda.synchronize()
    p.c.set_stream(st.cuda_stream)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        for f in calls:
            f()
    return g


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("past,m", [(0, 64), (10, 70), (64, 1), (70, 130)])
def test_fork_inside_a_chunk_ends_its_appends(dtype, past, m):
    """A fork shares the chunk's pages: whatever is appended afterwards, by a call
    or by a recorded launch, may not reach them. Attention goes on."""
    p = Pair(dtype, 4, 2, 64, 64, 4, 300, seed=past + m)
    p.add([0, 2], [past, 5])
    p.c.extend([0, 2], [m, 3])
    k, v, q = p.rows(m + 3), p.rows(m + 3), p.rows(m + 3, 4)[0]
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    p.c.append(-1, k.data_ptr(), v.data_ptr())
    for s, lo, hi in ((0, 0, m), (2, m, m + 3)):
        p.k[s], p.v[s] = torch.cat([p.k[s], k[:, lo:hi]], 1), torch.cat([p.v[s], v[:, lo:hi]], 1)
    st = torch.cuda.Stream()
    kk, vv = k + 1, v + 1
    g = recorded(p, st, lambda: p.c.append(-1, kk.data_ptr(), vv.data_ptr()), lambda: p.c.attend(0, q.data_ptr(), out.data_ptr()))
    p.c.fork(0, [1, 3])
    for s in (1, 3):
        p.k[s], p.v[s] = p.k[0], p.v[0]
    with pytest.raises(binding.WhisperError) as e:
        p.c.append(-1, kk.data_ptr(), vv.data_ptr())
    assert e.value.status == binding.E_STATE
    for _ in range(2):
        out.fill_(7)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        p.check(out, q, [0, 2], [m, 3])
        p.check_rows([0, 1, 2, 3])
    p.attend([0, 2], [m, 3], q=q)
    p.add([3, 0, 1], [1, 2, 1])  # the next chunk may be appended again
    p.attend([3, 0, 1], [1, 2, 1])
    p.check_rows([0, 1, 2, 3])


def test_fork_before_the_append():
    """A copied page would miss the rows that are still to come: such a chunk
    can no longer be appended. A fork of a sequence without new positions leaves it."""
    p = Pair("bf16", 4, 2, 64, 64, 4, 300)
    p.add([0, 1], [40, 40])
    k, v = p.rows(70), p.rows(70)
    p.c.extend([1, 0], [0, 70])
    p.c.fork(1, [2])  # (listed, without new positions)
    p.k[2], p.v[2] = p.k[1], p.v[1]
    p.c.append(-1, k.data_ptr(), v.data_ptr())
    p.k[0], p.v[0] = torch.cat([p.k[0], k], 1), torch.cat([p.v[0], v], 1)
    p.check_rows([0, 1, 2])
    p.c.extend([0], [30])
    p.c.fork(0, [])  # no copy
    p.c.append(-1, k.data_ptr(), v.data_ptr())
    p.k[0], p.v[0] = torch.cat([p.k[0], k[:, :30]], 1), torch.cat([p.v[0], v[:, :30]], 1)
    p.check_rows([0])
    p.c.extend([0], [7])
    p.c.fork(0, [3])
    with pytest.raises(binding.WhisperError) as e:
        p.c.append(-1, k.data_ptr(), v.data_ptr())
    assert e.value.status == binding.E_STATE
    p.c.truncate([0, 3], [140, 140])
    p.k[3], p.v[3] = p.k[0], p.v[0]
    p.check_rows([0, 3])


@pytest.mark.parametrize("H,Hkv,D", HEADS)
def test_few_rows_keep_their_weights(H, Hkv, D):
    """bf16 caches: rows that the kernel of few rows takes lose nothing of their
    softmax weights but what fp32 sums lose; the output alone is rounded to bf16."""
    G = H // Hkv
    p = Pair("bf16", H, Hkv, D, 64, 4, 2500, seed=D + H)
    p.add([0, 1, 2, 3], [0, 63, 700, 2100])
    for m in (1, 5):
        counts = [m] * 4
        p.add([0, 1, 2, 3], counts)
        q = p.rows(4 * m, H)[0] * 1.5
        out = torch.empty_like(q)
        torch.cuda.synchronize()
        p.c.attend(0, q.data_ptr(), out.data_ptr())
        torch.cuda.synchronize()
        for s in range(4):
            k, v = (x[s][0].double().repeat_interleave(G, 1).transpose(0, 1) for x in (p.k, p.v))
            e = k.shape[1]
            qs = q[s * m: s * m + m].double().transpose(0, 1)
            hidden = torch.arange(e, device="cuda")[None] > torch.arange(e - m, e, device="cuda")[:, None]
            sc = (torch.matmul(qs, k.transpose(1, 2).contiguous()) * D ** -0.5).masked_fill(hidden, -math.inf)
            w = torch.softmax(sc, -1)
            ref, mean = torch.matmul(w, v), torch.matmul(w, v.abs())
            # a score: D products and sums in fp32; a weight: the hardware exponential 2^-21, and as two
            # bf16 numbers 2^-8 of 2^-8; sums over the positions in fp32 (Pair.check), the output rounded once
            es = (D + 4) * 2.0 ** -24 * D ** -0.5 * torch.matmul(qs.abs(), k.abs().transpose(1, 2).contiguous()).amax()
            rel = 4 * es + 2.0 ** -20 + 2 * e * 2.0 ** -24 + 2.0 ** -16
            err = (out[s * m: s * m + m].double().transpose(0, 1) - ref).abs()
            tol = 2.0 ** -8 * ref.abs() + rel * mean * (1 + 2.0 ** -8) + 1e-30
            assert (err <= tol).all(), (s, m, float((err / tol).max()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 5, 200])
def test_infinite_values_in_sight(dtype, D, m):
    """An infinite value makes its dim infinite in the rows that see it, with its
    sign, two of different signs make it no number; other dims and rows go on."""
    p = Pair(dtype, 4, 2, D, 32, 1, 700, seed=m)
    past = 300
    k, v = p.rows(past + m), p.rows(past + m)
    k *= 0.25  # weights of one size: none of them vanishes
    v[0, 40, 0, 3] = math.inf
    v[0, 131, 1, 7] = -math.inf
    v[0, 140, 1, 9], v[0, 250, 1, 9] = math.inf, -math.inf
    late = past + m // 2
    v[0, late, 0, 11] = -math.inf
    q = p.rows(m, 4)[0]
    for a, b in ((0, past), (past, past + m)):
        p.add([0], [b - a], k[:, a:b].contiguous(), v[:, a:b].contiguous())
    out = torch.empty_like(q)
    p.c.attend(0, q.data_ptr(), out.data_ptr())
    torch.cuda.synchronize()
    x = out.float()
    assert (x[:, :2, 3] == math.inf).all() and (x[:, 2:, 7] == -math.inf).all() and x[:, 2:, 9].isnan().all()
    assert (x[m // 2:, :2, 11] == -math.inf).all() and x[: m // 2, :2, 11].isfinite().all()
    keep = torch.ones(4, D, dtype=torch.bool, device="cuda")
    keep[:2, 3] = keep[2:, 7] = keep[2:, 9] = keep[:2, 11] = False
    assert x[:, keep].isfinite().all()
    p.v[0] = torch.where(p.v[0].float().isfinite(), p.v[0], torch.zeros_like(p.v[0]))
    p.c.truncate([0], [0])
    p.k[0], p.v[0], kk, vv = p.k[0][:, :0], p.v[0][:, :0], p.k[0].contiguous(), p.v[0].contiguous()
    for a, b in ((0, past), (past, past + m)):
        p.add([0], [b - a], kk[:, a:b].contiguous(), vv[:, a:b].contiguous())
    zero = p.attend([0], [m], q=q)
    p.check(torch.where(keep, out, zero), q, [0], [m])
