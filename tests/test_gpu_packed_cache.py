"""The packed cache on the GPU against plain float64: what appended rows become,
attention over it, forks, reordered sequences, recorded launches."""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import operators as O
from paper_2507_01021_amd import binding

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, binding.DTYPE_F32), "bf16": (torch.bfloat16, binding.DTYPE_BF16)}
HEADS = [(6, 6, 64), (8, 2, 64), (5, 1, 64), (32, 8, 128), (3, 3, 128), (24, 1, 128)]


def held(x, bits):
    """What a cache of `bits` makes of rows, in float64 on the GPU."""
    if not bits or x.numel() == 0:
        return x.double()
    return torch.from_numpy(O.packed(x.double().cpu().numpy(), bits)[0]).cuda()


class Pair:
    """A packed cache beside what its sequences stand for."""

    def __init__(self, dtype, bits, H, Hkv, D, P, max_seqs, max_positions, layers=1, n_pages=None, max_tokens=None, seed=0):
        self.t, code = DT[dtype]
        self.bits, self.H, self.Hkv, self.D, self.layers = bits, H, Hkv, D, layers
        n_pages = n_pages or max_seqs * (-(-max_positions // P))
        self.c = binding.Cache(code, layers, H, Hkv, D, P, n_pages, max_seqs, max_positions,
                               max_tokens or max_seqs * max_positions, bits=bits)
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        e = torch.empty(layers, 0, Hkv, D, dtype=torch.float64, device="cuda")
        self.k, self.v = ([e] * max_seqs for _ in range(2))

    def rows(self, n, heads=None):
        return torch.randn(self.layers, n, heads or self.Hkv, self.D, generator=self.g, device="cuda").to(self.t)

    def note(self, seqs, counts, k, v):
        at = 0
        hk, hv = held(k, self.bits), held(v, self.bits)
        for s, m in zip(seqs, counts):
            self.k[s] = torch.cat([self.k[s], hk[:, at: at + m]], 1)
            self.v[s] = torch.cat([self.v[s], hv[:, at: at + m]], 1)
            at += m

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
        self.note(seqs, counts, k, v)
        torch.cuda.synchronize()

    def cut(self, seqs, lens):
        self.c.truncate(seqs, lens)
        for s, n in zip(seqs, lens):
            self.k[s], self.v[s] = self.k[s][:, :n], self.v[s][:, :n]

    def reorder(self, seqs, src):
        self.c.reorder(seqs, src)
        k, v = list(self.k), list(self.v)
        for s, f in zip(seqs, src):
            self.k[s], self.v[s] = k[f], v[f]

    def check_rows(self, seqs):
        n = sum(self.k[s].shape[1] for s in seqs)
        ko = torch.full((self.layers, n + 1, self.Hkv, self.D), 7.0, dtype=self.t, device="cuda")
        vo = ko.clone()
        for l in range(self.layers):
            self.c.read(l, seqs, ko[l].data_ptr(), vo[l].data_ptr())
        torch.cuda.synchronize()
        for got, want in ((ko, self.k), (vo, self.v)):
            assert (got[:, n] == 7).all()
            assert np.array_equal(got[:, :n].double().cpu().numpy(), torch.cat([want[s] for s in seqs], 1).cpu().numpy(), equal_nan=True)

    def attend(self, seqs, counts, layer=0, q=None, scale=None, big=None):
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
        one = torch.finfo(self.t).eps / 2
        bf = self.t == torch.bfloat16
        for s, m in zip(seqs, counts):
            k, v = (x[s][layer].repeat_interleave(G, 1).transpose(0, 1) for x in (self.k, self.v))
            past = k.shape[1] - m
            for i0 in range(0, m, 512):
                i1 = min(m, i0 + 512)
                e = past + i1
                qs = q[at + i0: at + i1].double().transpose(0, 1)
                hidden = torch.arange(e, device="cuda")[None] > torch.arange(past + i0, past + i1, device="cuda")[:, None]
                sc = (torch.matmul(qs, k[:, :e].transpose(1, 2).contiguous()) * scale).masked_fill(hidden, -math.inf)
                w = torch.softmax(sc, -1)
                ref, mean = torch.matmul(w, v[:, :e]), torch.matmul(w, v[:, :e].abs())
                # Codes enter products with an offset: |number| below `top` steps, where a group's step is at most
                # 1.125 (8 bits: 2) times its range / 15 (255), its range at most twice its largest value or so:
                # so a product's terms are at most `top` steps, `lift` times the group's largest value
                # (143 / 15 * 1.125 in 4 bits with bf16; 255 or 15 steps of at most 2 or 1.125 / top ranges else).
                lift = 2 * 143 / 15 * 1.125 if self.bits == 4 and bf else 4.5
                most = torch.stack([x.abs().unflatten(-1, (-1, 64)).amax(-1) for x in (k[:, :e], v[:, :e])])
                kmost, vmost = (x.repeat_interleave(64, -1) for x in most)
                # a score: D products and sums of such terms in fp32, codes and the zeros' term
                es = 2 * (self.D + 8) * 2.0 ** -24 * scale * lift * torch.matmul(qs.abs(), kmost.transpose(1, 2).contiguous()).amax()
                # sums over the positions: a wave adds one product of 32 positions (two in bf16) per 128
                # positions and rescales, each 2^-24 of the sum of its terms, and those of a product 32 of them;
                # at most one wave takes them all
                steps = 64 + 3 * e / 32
                # weights: the hardware exponential 2^-20, twice a score's error up and down; in bf16 as two
                # numbers 2^-16, or rounded to one where a sequence has 128 rows
                one_number = bf and m * G >= 128
                rel = 4 * es + 2.0 ** -20 + (2.0 ** -16 if bf else 0) + (one if one_number else 0)
                tol = one * ref.abs() + (1 + one) * (rel * mean + 2 * steps * 2.0 ** -24 * lift * torch.matmul(w, vmost)) + 1e-30
                err = (out[at + i0: at + i1].double().transpose(0, 1) - ref).abs()
                bad = ~(err <= tol)
                assert not bad.any(), (s, m, past, float((err / tol).nan_to_num(1e9).max()), bad.nonzero()[0].tolist())
            at += m


BOTH = pytest.mark.parametrize("dtype,bits", [("f32", 4), ("f32", 8), ("bf16", 4), ("bf16", 8)])


@BOTH
@pytest.mark.parametrize("H,Hkv,D", HEADS)
@pytest.mark.parametrize("P", [32, 128])
def test_rows_come_back(dtype, bits, H, Hkv, D, P):
    p = Pair(dtype, bits, H, Hkv, D, P, 5, 500, layers=3)
    p.add([0, 3, 1], [1, 131, 64])
    p.check_rows([0, 1, 3])
    p.add([1, 0, 2], [63, 31, 1], one_by_one=True)
    p.add([3], [1])
    p.add([4, 0, 2], [5, 1, 1])
    p.check_rows([3, 2, 1, 0, 4])


@BOTH
def test_rows_of_every_size(dtype, bits):
    """Groups of all magnitudes, of one number, of zeros, of one sign, with ties, at
    the ends of the range, with numbers that are not finite; a bad group
    leaves its neighbours alone."""
    p = Pair(dtype, bits, 4, 4, 128, 64, 2, 700)
    n = 300
    for one_by_one in (False, True):
        k, v = (x * torch.exp2(torch.randint(-118, 120, (1, n, 4, 1), generator=p.g, device="cuda").float()).to(p.t)
                for x in (p.rows(n), p.rows(n)))
        for x in (k, v):
            x[0, 0], x[0, 1], x[0, 2] = 0, 1.5, -2.25
            x[0, 3] = x[0, 3].abs()
            x[0, 4] = (torch.arange(128, device="cuda") * 0.25 - 16).to(p.t)
            x[0, 5, 0, 7], x[0, 6, 1, 64], x[0, 7, 2, 127] = math.nan, math.inf, -math.inf
            x[0, 8, 3, 0], x[0, 9, 0, 1] = 2.0 ** 125, -torch.finfo(p.t).max
            x[0, 10] = 0
            x[0, 10, :, 9], x[0, 11, :, 70] = 2.0 ** 124, -2.0 ** 124
            x[0, 12] = 1e-38
            x[0, 13] = torch.where(torch.arange(128, device="cuda") % 2 == 0, 7.5, -7.5).to(p.t)
        if one_by_one:
            for i in range(40):
                p.add([1], [1], k[:, i: i + 1].contiguous(), v[:, i: i + 1].contiguous())
        else:
            p.add([0], [n], k, v)
        p.check_rows([0, 1])


@BOTH
@pytest.mark.parametrize("H,Hkv,D", HEADS)
@pytest.mark.parametrize("P", [32, 64, 256])
def test_one_token_per_sequence(dtype, bits, H, Hkv, D, P):
    p = Pair(dtype, bits, H, Hkv, D, P, 7, 700, seed=P)
    p.add([0, 1, 2, 3, 4, 5], [31, 32, 33, 447, 127, 640])
    seqs = [5, 0, 1, 2, 3, 6, 4]  # 6: its first token
    for _ in range(3):
        p.add(seqs, [1] * 7)
        p.attend(seqs, [1] * 7)
    p.check_rows(seqs)


@BOTH
@pytest.mark.parametrize("H,Hkv,D", HEADS)
@pytest.mark.parametrize("P", [32, 64])
def test_chunks(dtype, bits, H, Hkv, D, P):
    p = Pair(dtype, bits, H, Hkv, D, P, 6, 900, seed=P + 1)
    p.add([0, 1, 2], [100, 5, 300])
    seqs, counts = [3, 0, 2, 1, 4, 5], [257, 1, 64, 0, 16, 200]
    p.add(seqs, counts)
    p.attend(seqs, counts)
    p.add([3, 1], [7, 333])
    p.attend([3, 1], [7, 333])


@BOTH
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 64), (8, 2, 128)])
def test_chunks_on_either_side_of_a_choice_of_kernel(dtype, bits, H, Hkv, D):
    """Rows of a sequence and kv head around 4, 16, 32 and 192; tokens around 4 a
    tile, whose mean decides how a chunk is appended."""
    p = Pair(dtype, bits, H, Hkv, D, 64, 6, 1500, seed=3)
    p.add([0, 1, 2, 3, 4, 5], [700, 1, 33, 31, 64, 255])
    G = H // Hkv
    for rows in ([192, 188, 196, 4, 8, 16], [4, 8, 12, 16, 20, 32], [4, 4, 4, 4, 4, 4], [36, 128, 124, 64, 4, 192]):
        counts = [r // G for r in rows]
        p.add(list(range(6)), counts)
        p.attend(list(range(6)), counts)
    for counts in ([1, 2, 3, 4, 5, 6], [4, 4, 4, 4, 4, 4], [5, 5, 5, 5, 5, 5], [191, 193, 1, 1, 1, 1], [0, 0, 33, 0, 0, 0]):
        p.add(list(range(6)), counts)
        p.attend(list(range(6)), counts)
    p.check_rows(list(range(6)))


@pytest.mark.parametrize("dtype,bits,H,Hkv,D,lens", [
    ("bf16", 4, 8, 2, 128, [20000, 1, 4097]), ("bf16", 8, 20, 20, 64, [9000]), ("bf16", 4, 8, 8, 64, [7001, 3000]),
    ("f32", 4, 4, 1, 64, [12345, 700]), ("f32", 8, 2, 2, 128, [5000]), ("bf16", 4, 1, 1, 64, [50000])])
def test_long_contexts_are_cut_and_joined(dtype, bits, H, Hkv, D, lens):
    n = len(lens)
    p = Pair(dtype, bits, H, Hkv, D, 128, n, max(lens) + 100)
    p.add(list(range(n)), lens)
    for counts in ([1] * n, [3] * n, [17] * n):
        p.add(list(range(n)), counts)
        p.attend(list(range(n)), counts)


@BOTH
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("left_over", [True, False])
def test_what_is_hidden_does_not_enter(dtype, bits, D, left_over):
    """Groups of NaN at later positions of the chunk, and left over in freed
    pages, reach no row that does not see them; rows that do hold NaN."""
    p = Pair(dtype, bits, 4, 2, D, 32, 2, 600, n_pages=40)
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
            assert torch.isnan(out[m // 2 + 1:, :, :64].float()).all()
            if D == 128:  # the values' other group is whole
                assert torch.isfinite(out[m // 2 + 1: m - 1, :, 64:].float()).all()
        k0, v0 = p.k[0], p.v[0]
        p.k[0], p.v[0] = k0[:, : past + clean], v0[:, : past + clean]
        p.check(out[:clean], q, [0], [clean])
        p.k[0], p.v[0] = k0, v0


@BOTH
def test_strides_and_unaligned_rows(dtype, bits):
    H, Hkv, D = 4, 2, 64
    p = Pair(dtype, bits, H, Hkv, D, 64, 2, 400)
    for n in (75, 2):
        p.cut([0, 1], [0, 0])
        fused = torch.randn(n, (H + 2 * Hkv) * D + 8, generator=p.g, device="cuda").to(p.t)
        ld = fused.stride(0)
        q, k, v = fused[:, : H * D], fused[:, H * D: (H + Hkv) * D], fused[:, (H + Hkv) * D: (H + 2 * Hkv) * D]
        p.c.extend([1], [n])
        p.c.append(0, k.data_ptr(), v.data_ptr(), ld, ld)
        out = torch.full((n, H * D + 16), 7.0, dtype=p.t, device="cuda")
        p.c.attend(0, q.data_ptr(), out.data_ptr(), ld, out.stride(0))
        torch.cuda.synchronize()
        assert (out[:, H * D:] == 7).all()
        p.note([1], [n], k.reshape(1, n, Hkv, D), v.reshape(1, n, Hkv, D))
        p.check(out[:, : H * D].reshape(n, H, D), q.reshape(n, H, D), [1], [n])
        # an odd address and odd strides
        odd = torch.randn(n * 401 + 1, generator=p.g, device="cuda").to(p.t)
        ko = odd[1:].view(n, 401)[:, 3: 3 + Hkv * D]
        vo = odd[1:].view(n, 401)[:, 200: 200 + Hkv * D]
        p.c.extend([0], [n])
        p.c.append(0, ko.data_ptr(), vo.data_ptr(), 401, 401)
        p.note([0], [n], ko.reshape(1, n, Hkv, D), vo.reshape(1, n, Hkv, D))
        back = torch.zeros(2, n * 301 + 1, dtype=p.t, device="cuda")
        kb, vb = (b[1:].view(n, 301) for b in back)
        p.c.read(0, [0], kb.data_ptr(), vb.data_ptr(), 301, 301)
        torch.cuda.synchronize()
        assert torch.equal(kb[:, : Hkv * D].double().reshape(n, Hkv, D), p.k[0][0])
        assert torch.equal(vb[:, : Hkv * D].double().reshape(n, Hkv, D), p.v[0][0])
        assert not kb[:, Hkv * D:].any() and not back[:, 0].any()


@pytest.mark.parametrize("bits", [4, 8])
def test_scale_and_large_scores(bits):
    p = Pair("bf16", bits, 2, 2, 64, 32, 1, 300)
    p.add([0], [200])
    p.add([0], [5])
    p.attend([0], [5], scale=3.0)  # nearly one-hot weights
    p.attend([0], [5], scale=1e-4)  # nearly equal ones


@BOTH
def test_results_do_not_depend_on_pages(dtype, bits):
    outs = []
    for mess in (False, True):
        p = Pair(dtype, bits, 4, 2, 64, 32, 4, 600, n_pages=80, seed=3)
        if mess:
            p.c.extend([3, 2], [90, 40])
        k, v = (torch.randn(1, 600, 2, 64, generator=p.g, device="cuda").to(p.t) for _ in range(2))
        q = torch.randn(90, 4, 64, generator=p.g, device="cuda").to(p.t)
        p.add([0], [480], k[:, :480].contiguous(), v[:, :480].contiguous())
        got = []
        for lo, hi in ((480, 500), (500, 590)):  # few rows, many rows
            p.add([0], [hi - lo], k[:, lo:hi].contiguous(), v[:, lo:hi].contiguous())
            if mess and lo == 480:
                p.c.truncate([3, 2], [0, 0])
            if mess:
                p.c.compact()  # pages move while the chunk is current
            got.append(p.attend([0], [hi - lo], q=q[: hi - lo]))
        outs.append(torch.cat(got))
        p.check_rows([0])
    assert torch.equal(outs[0], outs[1])


@BOTH
@pytest.mark.parametrize("past", [1, 64, 229])
def test_forks_go_their_own_way(dtype, bits, past):
    p = Pair(dtype, bits, 4, 4, 64, 64, 6, 300, layers=2, seed=past)
    p.add([0], [past])
    p.c.fork(0, [1, 2, 5])
    for s in (1, 2, 5):
        p.k[s], p.v[s] = p.k[0], p.v[0]
    p.check_rows([0, 1, 2, 5])
    for step in range(2):
        p.add([5, 0, 1, 2], [1, 2, 1, 1])
        for l in (0, 1):
            p.attend([5, 0, 1, 2], [1, 2, 1, 1], layer=l)
    p.cut([1, 2], [past - 1, past + 1])
    p.add([1, 2, 0], [3, 1, 1])
    p.attend([1, 2, 0], [3, 1, 1], layer=1)
    p.check_rows([0, 1, 2, 5])
    p.cut([0], [0])
    p.c.compact()
    p.check_rows([1, 2, 5])


@pytest.mark.parametrize("dtype,bits", [("f32", 0), ("bf16", 0), ("bf16", 4), ("f32", 8)])
def test_reordered_beams_go_their_own_way(dtype, bits):
    """Steps of beams that continue one another at random, some given up, some in
    place, in caches of all kinds."""
    r = random.Random(bits)
    p = Pair(dtype, bits, 4, 2, 64, 32, 6, 300, layers=2, seed=bits, n_pages=70)
    p.add([0, 1], [61, 30])
    p.reorder([2, 3, 4, 5], [0, 0, 1, 1])
    p.check_rows(list(range(6)))
    for step in range(12):
        p.add(list(range(6)), [1] * 6)
        p.attend(list(range(6)), [1] * 6, layer=step % 2)
        seqs = r.sample(range(6), r.randint(1, 6))
        p.reorder(seqs, [r.randrange(6) for _ in seqs])
        if step % 5 == 4:
            p.c.compact()
        p.check_rows(list(range(6)))


def test_reorder_and_the_chunk():
    """A sequence of the chunk that becomes another one ends the chunk; one that others
    continue is not appended to any more; others, and sequences that stay, go on."""
    p = Pair("bf16", 4, 4, 2, 64, 32, 6, 300)
    p.add([0, 1, 2], [40, 5, 64])
    x = p.rows(20)

    def refused(f):
        with pytest.raises(binding.WhisperError) as e:
            f()
        assert e.value.status == binding.E_STATE

    k, v, q = p.rows(4), p.rows(4), p.rows(4, 4)[0]
    p.c.extend([0, 1], [3, 1])
    p.c.append(-1, k.data_ptr(), v.data_ptr())
    p.note([0, 1], [3, 1], k, v)
    p.reorder([3, 0], [2, 0])  # neither touches the chunk
    p.c.append(-1, k.data_ptr(), v.data_ptr())
    p.attend([0, 1], [3, 1], q=q)
    p.reorder([4], [0])  # shares the chunk's pages
    refused(lambda: p.c.append(-1, x.data_ptr(), x.data_ptr()))
    p.attend([0, 1], [3, 1], q=q)
    p.reorder([1], [2])  # the chunk's row is gone
    refused(lambda: p.c.attend(0, x.data_ptr(), x.data_ptr()))
    refused(lambda: p.c.append(-1, x.data_ptr(), x.data_ptr()))
    p.check_rows([0, 1, 2, 3, 4])
    p.add([4, 1, 0], [1, 2, 1])
    p.attend([4, 1, 0], [1, 2, 1])
    p.check_rows([0, 1, 2, 3, 4])


@pytest.mark.parametrize("n", [3, 12, 24, 64])
@pytest.mark.parametrize("bits", [0, 8])
def test_reorders_of_many_pages(bits, n):
    """Lists of changed pages of any length, with a chunk that they end: all sequences
    in a circle, then all but two as one."""
    p = Pair("bf16", bits, 2, 1, 64, 32, n, 800, n_pages=n * 26, seed=n)
    lens = [600 + 11 * (i % 10) for i in range(n)]
    p.add(list(range(n)), lens)
    p.add([0, 1], [1, 2])  # a chunk
    p.reorder(list(range(n)), [(i + 1) % n for i in range(n)])
    x = p.rows(4, 2)[0]
    for f in (lambda: p.c.append(-1, x.data_ptr(), x.data_ptr()), lambda: p.c.attend(0, x.data_ptr(), x.data_ptr())):
        with pytest.raises(binding.WhisperError) as e:
            f()
        assert e.value.status == binding.E_STATE
    p.check_rows(list(range(n)))
    p.add(list(range(n)), [1] * n)
    p.attend(list(range(n)), [1] * n)
    p.reorder(list(range(2, n)), [1] * (n - 2))
    p.check_rows(list(range(n)))
    for _ in range(2):
        p.add(list(range(n)), [3] * n)
        p.attend(list(range(n)), [3] * n)
    p.check_rows(list(range(n)))


def record(p, st, *calls):
    torch.cuda.synchronize()
    p.c.set_stream(st.cuda_stream)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        for f in calls:
            f()
    return g


@BOTH
def test_recorded_step_serves_later_chunks(dtype, bits):
    """append and attend in a graph, replayed for chunks of other lengths and
    sequences (few and many rows), with the program's own work between."""
    n = 70
    p = Pair(dtype, bits, 8, 4, 64, 32, 6, 3000, max_tokens=12000)
    p.add([0, 1, 2, 3, 4, 5], [100, 2500, 7, 1000, 31, 32])
    k, v = (torch.zeros(1, n, 4, 64, dtype=p.t, device="cuda") for _ in range(2))
    q, out = (torch.zeros(n, 8, 64, dtype=p.t, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    p.c.set_stream(st.cuda_stream)
    p.c.extend([0, 2], [1, 1])
    p.c.append(0, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    p.note([0, 2], [1, 1], k[:, :2], v[:, :2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        p.c.append(0, k.data_ptr(), v.data_ptr())
        p.c.attend(0, q.data_ptr(), out.data_ptr())
        with pytest.raises(binding.WhisperError) as e:
            p.c.reorder([0], [1])
        assert e.value.status == binding.E_STATE
    for seqs, counts in (([0, 2, 4, 5], [1, 1, 1, 1]), ([1, 3, 0], [1, 64, 5]), ([1, 5, 4, 3], [1, 1, 66, 2])):
        p.c.extend(seqs, counts)
        m = sum(counts)
        with torch.cuda.stream(st):
            for x in (k, v, q):
                x.copy_(torch.randn(x.shape, generator=p.g, device="cuda"))
            torch.cuda.synchronize()
            for _ in range(2):
                g.replay()
        torch.cuda.synchronize()
        p.note(seqs, counts, k[:, :m], v[:, :m])
        p.check(out[:m], q[:m], seqs, counts)
        p.c.set_stream(st.cuda_stream)
        p.check_rows(seqs)
        (torch.randn(64, 64, device="cuda") @ torch.randn(64, 64, device="cuda")).sum().item()


def test_two_recorded_caches_at_once():
    """Graphs of two caches, one of 4 and one of 8 bits, replayed on two streams beside
    each other for chunks of few and of many rows (200 and more of a sequence and kv
    head): neither's workspaces are the other's."""
    n, made = 130, []
    for bits in (4, 8):
        p = Pair("bf16", bits, 8, 4, 64, 64, 4, 3000, max_tokens=12000, seed=bits)
        p.add([0, 1, 2, 3], [100, 2500, 7, 1000])
        k, v = (torch.zeros(1, n, 4, 64, dtype=p.t, device="cuda") for _ in range(2))
        q, out = (torch.zeros(n, 8, 64, dtype=p.t, device="cuda") for _ in range(2))
        st = torch.cuda.Stream()
        p.c.set_stream(st.cuda_stream)
        p.c.extend([0], [0])
        g = record(p, st, lambda: p.c.append(0, k.data_ptr(), v.data_ptr()), lambda: p.c.attend(0, q.data_ptr(), out.data_ptr()))
        made.append((p, st, g, k, v, q, out))
    for seqs, counts in (([0, 2], [120, 10]), ([1, 3, 0], [101, 2, 20]), ([3, 2, 1, 0], [1, 1, 1, 1])):
        for p, st, g, k, v, q, out in made:
            for x in (k, v, q):
                x.copy_(torch.randn(x.shape, generator=p.g, device="cuda"))
        torch.cuda.synchronize()
        for p, st, g, k, v, q, out in made:
            p.c.extend(seqs, counts)
        for _ in range(3):
            for p, st, g, k, v, q, out in made:
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        m = sum(counts)
        for p, st, g, k, v, q, out in made:
            p.note(seqs, counts, k[:, :m], v[:, :m])
            p.check(out[:m], q[:m], seqs, counts)
            p.check_rows([0, 1, 2, 3])


@pytest.mark.parametrize("bits", [0, 4])
def test_replays_after_a_reorder(bits):
    """Recorded launches write nothing once the chunk's sequences are shared, and do
    nothing at all once one of them is another."""
    p = Pair("bf16", bits, 4, 2, 64, 32, 4, 300, seed=bits)
    p.add([0, 1], [40, 10])
    k, v, q = p.rows(6), p.rows(6), p.rows(6, 4)[0]
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    p.c.extend([0, 1], [5, 1])
    p.c.append(-1, k.data_ptr(), v.data_ptr())
    p.note([0, 1], [5, 1], k, v)
    st = torch.cuda.Stream()
    kk, vv = k + 1, v + 1
    g = record(p, st, lambda: p.c.append(-1, kk.data_ptr(), vv.data_ptr()), lambda: p.c.attend(0, q.data_ptr(), out.data_ptr()))
    p.reorder([2], [0])
    for _ in range(2):
        out.fill_(7)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        p.check(out, q, [0, 1], [5, 1])
        p.check_rows([0, 1, 2])
    p.reorder([0], [3])
    p.add([3], [60])  # from pages that were given up
    p.cut([3], [59])
    out.fill_(7)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        g.replay()
    torch.cuda.synchronize()
    assert (out == 7).all()
    p.check_rows([0, 1, 2, 3])


@BOTH
def test_outputs_in_place_of_queries(dtype, bits):
    p = Pair(dtype, bits, 8, 2, 64, 32, 3, 3000, seed=4)
    p.add([0, 1, 2], [2600, 70, 0])
    for counts in ([1, 5, 3], [40, 200, 1]):
        p.add([0, 1, 2], counts)
        q = p.rows(sum(counts), 8)[0]
        x = q.clone()
        p.c.attend(0, x.data_ptr(), x.data_ptr())
        torch.cuda.synchronize()
        p.check(x, q, [0, 1, 2], counts)


def test_other_stream():
    p = Pair("bf16", 4, 4, 4, 64, 32, 2, 300)
    p.add([0], [100])
    st = torch.cuda.Stream()
    p.c.set_stream(st.cuda_stream)
    with torch.cuda.stream(st):
        p.add([0], [40])
        p.attend([0], [40])
    p.c.set_stream(None)
    p.add([0], [3])
    p.attend([0], [3])


@pytest.mark.parametrize("bits", [4, 8])
def test_offsets_beyond_32_bits(bits):
    """Pages behind the first 4 GiB of a cache's memory, in its last layer; few and
    many rows."""
    H, D, P, layers = 8, 128, 256, 64
    n_pages = 330 if bits == 4 else 180
    c = binding.Cache(binding.DTYPE_BF16, layers, H, H, D, P, n_pages, 2, n_pages * P, 400, bits=bits)
    most = 400
    for i in range((n_pages - 10) * P // most):
        c.extend([0], [most])  # pages 0 .. n_pages - 11: more than 4 GiB
    assert (c.info(0)[1] - 1) * 2 * layers * H * (P * D * bits // 8 + 2 * P * D // 64) > 2 ** 32
    n = 300
    k, v, q = (torch.randn(n, H, D, device="cuda").bfloat16() for _ in range(3))
    hk, hv = held(k, bits), held(v, bits)
    out = torch.empty_like(q)
    at = 0
    for m in (100, 150, 1, 49):
        c.extend([1], [m])
        for layer in (0, layers - 1):
            c.append(layer, k[at:].data_ptr(), v[at:].data_ptr())
            c.attend(layer, q[at:].data_ptr(), out[at:].data_ptr())
        at += m
    torch.cuda.synchronize()
    s = torch.matmul(q.double().transpose(0, 1), hk.permute(1, 2, 0).contiguous()) * D ** -0.5
    s += torch.full((n, n), -math.inf, device="cuda").double().triu(1)
    ref = torch.matmul(torch.softmax(s, -1), hv.transpose(0, 1).contiguous()).transpose(0, 1)
    # weights and outputs rounded once each to bf16, values below 6; the rest as in Pair.check is below 2^-9
    assert (out.double() - ref).abs().max() <= 6 * (2 * 2.0 ** -8 + 2.0 ** -9)
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    c.read(layers - 1, [1], kb.data_ptr(), vb.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(kb.double(), hk) and torch.equal(vb.double(), hv)


@pytest.mark.parametrize("bits", [4, 8])
def test_packed_attention_is_that_of_the_values_it_stands_for(bits):
    """The same queries over a cache of bf16 that was given what the packed one
    reads out."""
    p = Pair("bf16", bits, 8, 4, 64, 64, 2, 700)
    p.add([0, 1], [300, 17])
    for counts in ([1, 1], [70, 40]):
        p.add([0, 1], counts)
        q = p.rows(sum(counts), 8)[0]
        a = p.attend([0, 1], counts, q=q)
        lens = [p.k[s].shape[1] for s in (0, 1)]
        c = binding.Cache(binding.DTYPE_BF16, 1, 8, 4, 64, 64, 30, 2, 700, 1400)
        old = [n - m for n, m in zip(lens, counts)]
        for lo, hi in (([0, 0], old), (old, lens)):
            kk, vv = (torch.cat([x[s][0, l:h] for s, l, h in zip((0, 1), lo, hi)]).bfloat16() for x in (p.k, p.v))
            c.extend([0, 1], [h - l for l, h in zip(lo, hi)])
            c.append(0, kk.data_ptr(), vv.data_ptr())
            torch.cuda.synchronize()
        b = torch.empty_like(q)
        c.attend(0, q.data_ptr(), b.data_ptr())
        torch.cuda.synchronize()
        p.check(b, q, [0, 1], counts)
        assert (a.double() - b.double()).abs().max() <= 2.0 ** -6
