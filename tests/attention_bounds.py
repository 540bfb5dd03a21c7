"""How far attention over a packed cache may be from its definition, per output, from
what is rounded on the way: no worst case over a whole call enters, so that a
weight rounded once too often, or one block of 32 positions that is missing, is
seen. (u = 2^-24; torch tensors, any device.)

Before its output is rounded, a row is off by at most the sum of
  scores       each is a sum of D products in fp32, taken as a random walk with four
               times its length: 4 u sqrt(D) |q * k| in fp32, where operands are code -
               zero. In bf16 codes enter as 128 + code or as code, and what they are
               too much leaves again: 4 u 8 |q| TOP step per group of 64. A weight is
               off by that share of itself.
  exponentials 2^-20 of a weight (the argument's own rounding included)
  weights      bf16: two numbers of 8 bits, 2^-16; or one, 2^-8
  sums         a wave adds 64 products at most to a sum before it is joined with
               others (ranges of more than 640 positions are cut): 4 u sqrt(64) of a
               product's terms, |value| in fp32, TOP steps in bf16
Weights' errors count twice, in the sum and in what it is divided by."""
import math

import torch

U = 2.0 ** -24
TOP = {("bf16", 4): 143, ("bf16", 8): 255}


def half_step(dtype):
    return torch.finfo({"bf16": torch.bfloat16, "f32": torch.float32}[dtype]).eps / 2


def attention(dtype, bits, q, k, v, k_step, v_step, past, scale, one_number=False):
    """Float64 attention of rows q [m][H][D] over k, v [past + m][Hkv][D] (float64, what the
    cache stands for; steps [past + m][Hkv][D / 64]). Returns outputs [H][m][D] and how far
    they may be off before they are rounded."""
    m, H, D = q.shape
    G = H // k.shape[1]
    k, v, k_step, v_step = (x.double().repeat_interleave(G, 1).transpose(0, 1).contiguous() for x in (k, v, k_step, v_step))
    q = q.double().transpose(0, 1).contiguous()
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    hidden = torch.arange(past + m, device=q.device)[None] > torch.arange(past, past + m, device=q.device)[:, None]
    w = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
    if dtype == "f32":
        es = 4 * U * scale * math.sqrt(D) * torch.matmul(q.square(), k.square().transpose(1, 2).contiguous()).sqrt()
        terms = v.abs()
    else:
        norms = q.unflatten(-1, (-1, 64)).square().sum(-1).sqrt()
        es = 4 * U * scale * 8 * TOP[dtype, bits] * torch.matmul(norms, k_step.transpose(1, 2).contiguous())
        terms = TOP[dtype, bits] * v_step.repeat_interleave(64, -1)
    each = 2.0 ** -20 + (0 if dtype == "f32" else half_step("bf16") if one_number else 2.0 ** -16)
    out = torch.matmul(w, v)
    # sum of w (es + each) (|v| + |out|), and the sums' own
    off = torch.matmul(w * (es + each), v.abs()) + (w * (es + each)).sum(-1, keepdim=True) * out.abs()
    return out, off + 4 * U * 8 * torch.matmul(w, terms)


def zeros_probe(dtype, bits, n, m, H, Hkv, D, seed):
    """Rows q, k, v on the CPU that make the zeros' term of the scores (minus zero + offset times a
    query's sum) large against the scores, which are all 0: queries of one sign, their dims
    in equal pairs, and keys of +- a size in turn, or of 0, in turn. Values say which keys they are of."""
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(m, H, D // 2, generator=g).abs().repeat_interleave(2, -1)
    one = (torch.arange(n) % 2).float()[:, None, None]
    k = one * ((80.0 if bits == 4 else 1000.0) * (1 - 2 * (torch.arange(D) % 2)))[None, None] * torch.ones(1, Hkv, 1)
    return q.to(t), k.to(t), (one * torch.ones(1, Hkv, D)).to(t)


def faults(dtype, got, out, off):
    """What is wrong with outputs got [H][m][D] (text; empty: nothing): one of them is
    further off than its bound and one rounding, or (bf16) more of them are not the
    rounded reference than bounds of that size bring about."""
    got, half = got.double(), half_step(dtype)
    tol = off + half * (out.abs() + off)
    err = (got - out).abs()
    bad = ~(err <= tol)  # (both may be 0)
    if bad.any():
        return "%d outputs are up to %.3g times their bounds off" % (int(bad.sum()), float((err / tol)[bad].nan_to_num(math.inf).max()))
    if dtype == "bf16":
        # an output is another than the rounded reference if a border between two
        # roundings lies within `off`; of a spacing of 2 half |out| / 2 .. 2 half |out|
        share = (2 * off / (half * out.abs())).clamp(max=1.0)
        expected = float(share.sum())
        differ = int((got != out.to(torch.bfloat16).double()).sum())
        if differ > expected + 6 * math.sqrt(expected) + 3:
            return "%d of %d outputs are not the rounded reference, %.0f expected at most" % (differ, got.numel(), expected)
    return ""
