"""Queries and outputs of attention over packed caches at addresses and strides that
are multiples of 16 bytes and of no more."""
import pytest

torch = pytest.importorskip("torch")

from paper_2507_01021_amd import binding

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, binding.DTYPE_F32), "bf16": (torch.bfloat16, binding.DTYPE_BF16)}


@pytest.mark.parametrize("dtype,bits", [("f32", 4), ("f32", 8), ("bf16", 4), ("bf16", 8)])
@pytest.mark.parametrize("H,Hkv,D", [(6, 6, 64), (8, 2, 128), (32, 1, 64)])
def test_rows_aligned_to_16_bytes(dtype, bits, H, Hkv, D):
    t, code = DT[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(D)
    c = binding.Cache(code, 1, H, Hkv, D, 32, 40, 2, 600, 600, bits=bits)
    piece = 16 // t.itemsize
    for past, m in ((37, 1), (100, 9), (0, 250)):
        c.truncate([0, 1], [0, 0])
        for counts in ([past, 5], [m, 1]):
            n = sum(counts)
            k, v = (torch.randn(n, Hkv * D, generator=g, device="cuda").to(t) for _ in range(2))
            c.extend([0, 1], counts)
            c.append(0, k.data_ptr(), v.data_ptr())
            torch.cuda.synchronize()
        n, width = m + 1, H * D
        q = torch.randn(n, width, generator=g, device="cuda").to(t)
        want = torch.empty_like(q)
        c.attend(0, q.data_ptr(), want.data_ptr())
        torch.cuda.synchronize()
        for first, ld in ((1, width), (0, width + piece), (1, width + piece), (3, width + 3 * piece)):
            flat = torch.full((2, first * piece + n * ld), 7.0, device="cuda", dtype=t)
            rows = [x[first * piece:].view(n, ld)[:, :width] for x in flat]
            rows[0].copy_(q)
            torch.cuda.synchronize()
            assert rows[0].data_ptr() % 32 == first * 16 % 32
            c.attend(0, rows[0].data_ptr(), rows[1].data_ptr(), ld, ld)
            torch.cuda.synchronize()
            assert torch.equal(rows[1], want)
            rows[1].fill_(7.0)
            assert (flat[1] == 7.0).all()  # nothing between the rows
