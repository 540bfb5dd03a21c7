"""Attention over packed caches whose values are near the ends of what a group
holds (magnitudes below 2^125): weighted sums of many of them do not fit fp32,
their weighted mean does."""
import math

import pytest

torch = pytest.importorskip("torch")

from oracle import operators as O
from paper_2507_01021_amd import binding

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, binding.DTYPE_F32), "bf16": (torch.bfloat16, binding.DTYPE_BF16)}


def held(x, bits):
    return torch.from_numpy(O.packed(x.double().cpu().numpy(), bits)[0]).cuda()


class Rows:
    """One sequence of a cache, and what it stands for."""

    def __init__(self, dtype, bits, H, Hkv, D, seed):
        self.t, code = DT[dtype]
        self.bits, self.H, self.Hkv, self.D = bits, H, Hkv, D
        self.c = binding.Cache(code, 1, H, Hkv, D, 64, 100, 1, 6400, 6400, bits=bits)
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def randn(self, *shape):
        return torch.randn(*shape, self.D, generator=self.g, device="cuda")

    def run(self, k, v, past):
        """Appends rows, the first `past` of them as a chunk of their own, and attends for
        the others; returns outputs, reference and the weighted mean of magnitudes."""
        k, v = k.to(self.t), v.to(self.t)
        n, scale = len(k), self.D ** -0.5
        self.c.truncate([0], [0])
        for lo, hi in ((0, past), (past, n)):
            if hi > lo:
                a, b = k[lo:hi].contiguous(), v[lo:hi].contiguous()
                self.c.extend([0], [hi - lo])
                self.c.append(0, a.data_ptr(), b.data_ptr())
                torch.cuda.synchronize()
        q = self.randn(n - past, self.H).to(self.t)
        out = torch.empty_like(q)
        self.c.attend(0, q.data_ptr(), out.data_ptr())
        torch.cuda.synchronize()
        G = self.H // self.Hkv
        hk, hv = (held(x, self.bits).repeat_interleave(G, 1).transpose(0, 1) for x in (k, v))
        s = torch.matmul(q.double().transpose(0, 1), hk.transpose(1, 2).contiguous()) * scale
        hidden = torch.arange(n, device="cuda")[None] > torch.arange(past, n, device="cuda")[:, None]
        w = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
        return out.double().transpose(0, 1), torch.matmul(w, hv), torch.matmul(w, hv.abs())

    def check(self, out, ref, mean, tokens):
        """Outputs rounded once; scores, exponentials and sums (of codes with an offset of up to 128,
        16 times a group's values) a few 2^-24 each; in bf16 weights as two numbers, or,
        from 192 rows of a kv head on, one."""
        one = torch.finfo(self.t).eps / 2
        bf = self.t == torch.bfloat16
        rel = (2.0 ** -13 if bf else 2.0 ** -18) + (one if bf and tokens * (self.H // self.Hkv) >= 192 else 0)
        assert torch.isfinite(out).all(), int((~torch.isfinite(out)).sum())
        assert ((out - ref).abs() <= one * ref.abs() + (1 + one) * rel * mean).all()


@pytest.mark.parametrize("dtype,bits", [("f32", 4), ("f32", 8), ("bf16", 4), ("bf16", 8)])
@pytest.mark.parametrize("H,Hkv,D", [(8, 2, 64), (2, 2, 128)])
@pytest.mark.parametrize("past,m", [(0, 1), (1, 1), (15, 1), (299, 1), (40, 30), (0, 300), (5000, 1), (5000, 200)])
def test_values_near_the_ends_of_the_range(dtype, bits, H, Hkv, D, past, m):
    """One token, drafts, prompts (in bf16 unpacked first), and ranges that are cut. A
    head of ordinary values beside one of large ones; ordinary values afterwards."""
    p = Rows(dtype, bits, H, Hkv, D, past + m)
    n = past + m
    for e in (78, 84, 119, 121, 124):
        k, v = p.randn(n, Hkv), p.randn(n, Hkv)
        v[:, 0] = (v[:, 0] * 0.4).clamp(-1, 1)
        v[:, 0, 0::8], v[:, 0, 1::8] = 1, -1  # in every group, at every position
        v[:, 0] *= 2.0 ** e
        p.check(*p.run(k, v, past), m)
        v[:, 0, :64] = 2.0 ** e  # all of a group alike
        p.check(*p.run(torch.zeros_like(k), v, past), m)  # equal weights
    p.check(*p.run(p.randn(n, Hkv), p.randn(n, Hkv), past), m)
    v = p.randn(n, Hkv) * 2.0 ** -30
    p.check(*p.run(p.randn(n, Hkv), v, past), m)
