"""The bounds that attention over a packed cache is held to: they let arithmetic pass
that rounds as the kernels say they do, and none that rounds once more or leaves
positions out (no GPU needed)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import attention_bounds as B
from oracle import operators as O


def made(dtype, bits, n, m=1, H=4, Hkv=2, D=64, seed=0):
    g = torch.Generator().manual_seed(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = [torch.randn(n, Hkv, D, generator=g).to(t) for _ in range(2)]
    held = [O.packed(y.double().numpy(), bits) for y in x]
    (k, ks), (v, vs) = [[torch.from_numpy(a) for a in h[:2]] for h in held]
    return torch.randn(m, H, D, generator=g).to(t), k, v, ks, vs


def computed(dtype, q, k, v, past, scale, weights=None, queries=None, leave_out=(0, 0)):
    """Attention in fp32 (float64 sums, rounded where the kernels round), as they may do it."""
    m, H, D = q.shape
    G = H // k.shape[1]
    k, v = (x.repeat_interleave(G, 1).transpose(0, 1) for x in (k, v))
    q = (q if queries is None else queries(q.float())).double().transpose(0, 1)
    s = (torch.matmul(q, k.transpose(1, 2)) * scale).float().double()
    hidden = torch.arange(past + m)[None] > torch.arange(past, past + m)[:, None]
    s = s.masked_fill(hidden, -math.inf)
    s[..., leave_out[0]: leave_out[1]] = -math.inf
    p = torch.exp(s - s.amax(-1, keepdim=True)).float()
    l = p.double().sum(-1, keepdim=True)
    p = p.double() if weights is None else weights(p).double()
    out = (torch.matmul(p, v) / l).float()
    return out.to(torch.bfloat16) if dtype == "bf16" else out


def bf16(x):
    return x.to(torch.bfloat16).float()


def bf16_twice(x):
    return bf16(x) + bf16(x - bf16(x))


LENGTHS = [38, 300, 4097]


@pytest.mark.parametrize("dtype,bits", [("f32", 4), ("f32", 8), ("bf16", 4), ("bf16", 8)])
@pytest.mark.parametrize("n", LENGTHS)
@pytest.mark.parametrize("m", [1, 5])
def test_what_the_bounds_let_pass(dtype, bits, n, m):
    q, k, v, ks, vs = made(dtype, bits, n, m)
    out, off = B.attention(dtype, bits, q, k, v, ks, vs, n - m, 0.125)
    got = computed(dtype, q, k, v, n - m, 0.125, weights=bf16_twice if dtype == "bf16" else None)
    assert B.faults(dtype, got, out, off) == ""
    if dtype == "bf16":
        out, off = B.attention(dtype, bits, q, k, v, ks, vs, n - m, 0.125, one_number=True)
        assert B.faults(dtype, computed(dtype, q, k, v, n - m, 0.125, weights=bf16), out, off) == ""


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n", LENGTHS)
def test_fp32_is_fp32(bits, n):
    q, k, v, ks, vs = made("f32", bits, n, 5)
    out, off = B.attention("f32", bits, q, k, v, ks, vs, n - 5, 0.125)
    for how in (dict(weights=bf16), dict(queries=bf16)):
        assert B.faults("f32", computed("f32", q, k, v, n - 5, 0.125, **how), out, off), how
    assert B.faults("f32", bf16(computed("f32", q, k, v, n - 5, 0.125)), out, off)


@pytest.mark.parametrize("bits,n", [(4, 38), (4, 300), (8, 38), (8, 300), (8, 4097)])
def test_weights_in_bf16_are_two_numbers(bits, n):
    """(Over 4097 positions in 4 bits, what is rounded away of so many weights is below
    the rounding of sums of 128 + code.)"""
    q, k, v, ks, vs = made("bf16", bits, n, 8, H=8)
    out, off = B.attention("bf16", bits, q, k, v, ks, vs, n - 8, 0.125)
    assert B.faults("bf16", computed("bf16", q, k, v, n - 8, 0.125, weights=bf16), out, off)


@pytest.mark.parametrize("dtype,bits", [("f32", 4), ("f32", 8), ("bf16", 4), ("bf16", 8)])
@pytest.mark.parametrize("n", LENGTHS + [20000, 50000])
def test_a_block_that_is_missing_is_seen(dtype, bits, n):
    q, k, v, ks, vs = made(dtype, bits, n, 1, H=2, Hkv=1)
    out, off = B.attention(dtype, bits, q, k, v, ks, vs, n - 1, 0.125)
    two = bf16_twice if dtype == "bf16" else None
    assert B.faults(dtype, computed(dtype, q, k, v, n - 1, 0.125, weights=two), out, off) == ""
    for at in (0, (n // 2) & ~31, (n - 33) & ~31):
        got = computed(dtype, q, k, v, n - 1, 0.125, weights=two, leave_out=(at, at + 32))
        assert B.faults(dtype, got, out, off), at


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("numbers", [2, 3])
def test_a_sum_of_queries_is_three_numbers(bits, numbers):
    """The zeros' term with a query's sum as so many bf16 numbers."""
    q, k, v = B.zeros_probe("bf16", bits, 64, 5, 4, 2, 64, 0)
    (k, ks, kz), (v, vs, _) = [[torch.from_numpy(a) for a in O.packed(x.double().numpy(), bits)] for x in (k, v)]
    out, off = B.attention("bf16", bits, q, k, v, ks, vs, 59, 0.125)
    total = q.double().sum(-1).transpose(0, 1)
    left = total.clone()
    for _ in range(numbers):
        left -= left.to(torch.bfloat16).double()
    k, v, ks, kz = (x.repeat_interleave(2, 1).transpose(0, 1) for x in (k, v, ks, kz))
    s = torch.matmul(q.double().transpose(0, 1), k.transpose(1, 2)) + left[..., None] * ((kz + (128 if bits == 4 else 0)) * ks).transpose(1, 2)
    hidden = torch.arange(64)[None] > torch.arange(59, 64)[:, None]
    got = torch.matmul(torch.softmax((s * 0.125).masked_fill(hidden, -math.inf), -1), v).to(torch.bfloat16)
    assert (B.faults("bf16", got, out, off) == "") == (numbers == 3)
