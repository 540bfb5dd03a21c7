"""Attention over packed caches against float64, held to bounds that see a weight
rounded once more or a block left out (test_attention_bounds.py shows that they
do), and by values that say which blocks were counted."""
import pytest

torch = pytest.importorskip("torch")

import attention_bounds as B
from oracle import operators as O
from paper_2507_01021_amd import binding

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, binding.DTYPE_F32), "bf16": (torch.bfloat16, binding.DTYPE_BF16)}
BOTH = pytest.mark.parametrize("dtype,bits", [("f32", 4), ("f32", 8), ("bf16", 4), ("bf16", 8)])


def held(x, bits):
    return [torch.from_numpy(a).cuda() for a in O.packed(x.double().cpu().numpy(), bits)[:2]]


# tokens by query heads a kv head: kernels of up to 4 rows (bf16), of 16, and of 128 (bf16, unpacked first)
@BOTH
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 64), (8, 2, 128), (20, 20, 64), (16, 1, 64)])
@pytest.mark.parametrize("past,m", [(0, 1), (37, 1), (299, 1), (640, 2), (1000, 1), (63, 5), (450, 17), (200, 200), (700, 48)])
def test_within_the_bounds(dtype, bits, H, Hkv, D, past, m):
    t, code = DT[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(past * 1000 + m)
    n = past + m
    c = binding.Cache(code, 1, H, Hkv, D, 64, 40, 2, 1100, 2200, bits=bits)
    k, v, q = (torch.randn(n, h, D, generator=g, device="cuda").to(t) for h in (Hkv, Hkv, H))
    for lo, hi in ((0, past), (past, n)):
        if hi > lo:
            a, b = k[lo:hi].contiguous(), v[lo:hi].contiguous()
            c.extend([1], [hi - lo])
            c.append(0, a.data_ptr(), b.data_ptr())
            torch.cuda.synchronize()
    q = q[past:].contiguous()
    out = torch.empty_like(q)
    c.attend(0, q.data_ptr(), out.data_ptr())
    torch.cuda.synchronize()
    one = dtype == "bf16" and m * (H // Hkv) >= 192
    (hk, ks), (hv, vs) = held(k, bits), held(v, bits)
    ref, off = B.attention(dtype, bits, q, hk, hv, ks, vs, past, D ** -0.5, one)
    assert B.faults(dtype, out.transpose(0, 1), ref, off) == ""


@pytest.mark.parametrize("dtype,bits,H,Hkv,D,n", [
    ("bf16", 4, 2, 2, 64, 4097), ("bf16", 4, 8, 2, 128, 7001), ("bf16", 4, 1, 1, 64, 20000), ("bf16", 4, 1, 1, 64, 50000),
    ("bf16", 8, 4, 4, 64, 9000), ("f32", 4, 4, 1, 64, 12345), ("f32", 8, 2, 2, 128, 5000)])
@pytest.mark.parametrize("m", [1, 3, 17])
def test_long_contexts_within_the_bounds(dtype, bits, H, Hkv, D, n, m):
    t, code = DT[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(n + m)
    c = binding.Cache(code, 1, H, Hkv, D, 128, 400, 1, 51200, 51200, bits=bits)
    k, v = (torch.randn(n, Hkv, D, generator=g, device="cuda").to(t) for _ in range(2))
    q = torch.randn(m, H, D, generator=g, device="cuda").to(t)
    for lo, hi in ((0, n - m), (n - m, n)):
        a, b = k[lo:hi].contiguous(), v[lo:hi].contiguous()
        c.extend([0], [hi - lo])
        c.append(0, a.data_ptr(), b.data_ptr())
        torch.cuda.synchronize()
    out = torch.empty_like(q)
    c.attend(0, q.data_ptr(), out.data_ptr())
    torch.cuda.synchronize()
    (hk, ks), (hv, vs) = held(k, bits), held(v, bits)
    ref, off = B.attention(dtype, bits, q, hk, hv, ks, vs, n - m, D ** -0.5)
    assert B.faults(dtype, out.transpose(0, 1), ref, off) == ""


@BOTH
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 64), (8, 2, 128)])
@pytest.mark.parametrize("n,m", [(64, 1), (64, 5), (300, 17), (400, 200)])
def test_the_zeros_term_is_whole(dtype, bits, H, Hkv, D, n, m):
    code = DT[dtype][1]
    q, k, v = (x.cuda() for x in B.zeros_probe(dtype, bits, n, m, H, Hkv, D, n + m))
    c = binding.Cache(code, 1, H, Hkv, D, 32, 20, 1, 600, 600, bits=bits)
    for lo, hi in ((0, n - m), (n - m, n)):
        a, b = k[lo:hi].contiguous(), v[lo:hi].contiguous()
        c.extend([0], [hi - lo])
        c.append(0, a.data_ptr(), b.data_ptr())
        torch.cuda.synchronize()
    out = torch.empty_like(q)
    c.attend(0, q.data_ptr(), out.data_ptr())
    torch.cuda.synchronize()
    (hk, ks), (hv, vs) = held(k, bits), held(v, bits)
    ref, off = B.attention(dtype, bits, q, hk, hv, ks, vs, n - m, D ** -0.5, dtype == "bf16" and m * (H // Hkv) >= 192)
    assert B.faults(dtype, out.transpose(0, 1), ref, off) == ""


@BOTH
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("n", [1, 33, 512, 513, 640, 4097, 20011])
def test_every_block_counts_once(dtype, bits, G, n):
    """Keys of zeros, so that all visible positions weigh alike, and in every block of 32
    a value in a dim (of a head, of a layer) of its own."""
    t, code = DT[dtype]
    Hkv, D = 2, 128
    H, per_layer = G * Hkv, Hkv * D
    layers = -(-(-(-(n + 200) // 32)) // per_layer)
    c = binding.Cache(code, layers, H, Hkv, D, 64, 700, 2, 21000, 21000, bits=bits)
    one = float(O.packed(torch.eye(64)[:1].numpy(), bits)[0].max())
    c.extend([1], [100])  # (beside the chunk's sequence)
    have = 0
    for m in (n, 1, 3, 17, 150):
        if m == n:
            c.extend([0], [m])
        else:
            c.extend([1, 0], [2, m])
        rows = m if m == n else m + 2
        values = torch.zeros(layers, rows, Hkv, D, device="cuda", dtype=t)
        at = torch.arange(have, have + m, device="cuda")
        b = at // 32
        values.view(layers, rows, per_layer)[b // per_layer, torch.arange(rows - m, rows, device="cuda"), b % per_layer] = 1
        keys = torch.zeros_like(values)
        c.append(-1, keys.data_ptr(), values.data_ptr())
        have += m
        q = torch.randn(rows, H, D, device="cuda").to(t)
        out = torch.empty_like(q)
        for layer in range(layers):
            c.attend(layer, q.data_ptr(), out.data_ptr())
            torch.cuda.synchronize()
            got = out[rows - m:].double().view(m, Hkv, G, D)
            ids = torch.arange(layer * per_layer, (layer + 1) * per_layer, device="cuda")
            seen = (at[:, None] + 1 - ids * 32).clamp(0, 32)  # of each block, by each row
            want = (seen * one / (at[:, None] + 1)).double().view(m, Hkv, 1, D)
            # (a position more or less is 1 / 32 of a block's; equal weights, sums of 32, one rounding: 2^-8 and little else)
            assert ((got - want).abs() <= want * 2.0 ** -7 + 2.0 ** -7 * one * 32 / (at + 1).double().view(m, 1, 1, 1) / 32).all(), (m, layer)
