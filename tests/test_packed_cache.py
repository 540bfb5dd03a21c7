"""The packed cache and reordered sequences on a handle without a device (no GPU
needed): the quantiser's oracle, the book, refusals."""
import os
import random
from fractions import Fraction

import numpy as np
import pytest

from oracle import operators as O
from paper_2507_01021_amd import binding

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH), reason="library not built")


def cache(**kw):
    p = dict(dtype=binding.DTYPE_BF16, n_layer=2, n_head=4, n_kv_head=2, head_size=64, page_size=32, n_pages=8, max_seqs=6,
             max_positions=200, max_tokens=300, device=binding.NO_DEVICE)
    p.update(kw)
    return binding.Cache(**p)


def refused(status, f, *a, **kw):
    with pytest.raises(binding.WhisperError) as e:
        f(*a, **kw)
    assert e.value.status == status, e.value
    assert str(e.value)


def bf16(x):
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("wide", [False, True])
def test_oracle_against_rational_numbers(bits, wide):
    """Step, zero and values of every group by exact arithmetic; the values are bf16
    numbers at most half a step away."""
    r = np.random.default_rng(bits)
    x = (r.standard_normal((40, 64)) * np.exp2(r.integers(-110, 120, (40, 1)))).astype(np.float32)
    x[:8] = np.abs(x[:8])
    x[8:12] = -np.abs(x[8:12])
    x[12] = 0
    x[13] = 1.5
    x[14] = np.arange(64) * 0.25 - 3.75  # ties of codes
    if not wide:
        x = bf16(x)
    v, step, zero = O.packed(x, bits)
    top, digits = 2 ** bits - 1, 4 if bits == 4 else 1
    for row, got, s, z in zip(x, v, step[:, 0], zero[:, 0]):
        row = [Fraction(float(y)) for y in row]
        lo, hi = min(0, *row), max(0, *row)
        spread = Fraction(float(np.float32(float(hi - lo))))
        s, z = Fraction(float(s)), int(z)
        assert s * top >= spread and s >= Fraction(1, 2 ** 100)
        m = s
        while m >= 2 ** digits:
            m /= 2
        while m < 2 ** (digits - 1):
            m *= 2
        assert m.denominator == 1
        if s > Fraction(1, 2 ** 100):  # the next smaller step would not do
            less = s - s / m if m > 2 ** (digits - 1) else s - s / m / 2
            assert less * top < spread
        assert z == round(-lo / s)
        for y, g in zip(row, got):
            want = (min(max(round(y / s) + z, 0), top) - z) * s
            assert Fraction(float(g)) == want and abs(want - y) <= s / 2
    assert (bf16(v) == v).all()


def test_oracle_of_what_is_not_a_number():
    x = np.ones((5, 128))
    x[0, 3], x[1, 70], x[2, 0], x[3, 127] = np.nan, np.inf, -2.0 ** 125, 2.0 ** 124
    v, _, _ = O.packed(x, 4)
    assert np.isnan(v[0, :64]).all() and np.isnan(v[1, 64:]).all() and np.isnan(v[2, :64]).all()
    assert np.isfinite(v[0, 64:]).all() and np.isfinite(v[3]).all()


def test_create_packed_refuses():
    for bits in (-1, 1, 2, 3, 5, 16):
        refused(binding.E_INVAL, cache, bits=bits)
    refused(binding.E_INVAL, cache, bits=4, head_size=80)
    for bits in (0, 4, 8):
        assert cache(bits=bits).info(0) == (0, 0, 8)
    lib = binding.load()
    assert lib.whisper_cache_create_packed(None, 4, 0, None) == binding.E_INVAL
    assert lib.whisper_cache_reorder(None, None, None, 0) == binding.E_INVAL


@pytest.mark.parametrize("bits", [4, 8])
def test_calls_check_their_arguments_first(bits):
    c = cache(bits=bits)
    c.extend([0], [1])
    ok = 4096
    refused(binding.E_INVAL, c.append, 2, ok, ok)
    refused(binding.E_INVAL, c.append, 0, 0, ok)
    refused(binding.E_INVAL, c.append, 0, ok, ok + 1)
    refused(binding.E_INVAL, c.attend, 0, ok + 2, ok)
    refused(binding.E_INVAL, c.attend, 0, ok, ok, q_stride=260)
    refused(binding.E_STATE, c.append, 0, ok, ok)  # no device
    refused(binding.E_STATE, c.attend, 0, ok, ok)
    refused(binding.E_STATE, c.read, 0, [0], ok, ok)


def test_reorder_checks_its_lists():
    c = cache()
    c.extend([0, 1], [40, 3])
    refused(binding.E_INVAL, c.reorder, [1, 1], [0, 0])
    refused(binding.E_INVAL, c.reorder, [1], [0, 0])
    refused(binding.E_CAPACITY, c.reorder, [6], [0])
    refused(binding.E_CAPACITY, c.reorder, [0], [6])
    refused(binding.E_CAPACITY, c.reorder, [-1], [0])
    refused(binding.E_CAPACITY, c.reorder, [0], [-1])
    refused(binding.E_INVAL, c.reorder, list(range(7)), [0] * 7)
    lib = binding.load()
    assert lib.whisper_cache_reorder(c.h, None, None, 1) == binding.E_INVAL
    s = np.zeros(1, np.int32)
    assert lib.whisper_cache_reorder(c.h, binding._ptr(s, binding.C.c_int32), None, 1) == binding.E_INVAL
    assert [c.info(s) for s in (0, 1, 2)] == [(40, 2, 5), (3, 1, 5), (0, 0, 5)]
    c.reorder([], [])


def test_reorder_shares_pages_and_the_last_holder_writes_in_place():
    c = cache()
    c.extend([0, 1], [40, 33])  # 2 pages each
    c.reorder([0, 1, 2], [1, 1, 0])
    assert [c.info(s)[:2] for s in (0, 1, 2)] == [(33, 2), (33, 2), (40, 2)]
    assert c.info(0)[2] == 4  # nothing was copied
    c.extend([0, 1, 2], [1, 1, 1])  # one copy for the two that share, none for the other
    assert c.info(0)[2] == 3
    c.reorder([0, 1], [1, 0])  # places changed: the same pages
    c.reorder([2], [3])  # an empty one: given up
    assert c.info(2) == (0, 0, 5)
    c.reorder([0, 1], [5, 5])
    assert c.info(0) == (0, 0, 8)


def test_random_reorders_against_a_plain_book():
    r = random.Random(7)
    c = cache(n_pages=40, max_seqs=7, max_positions=400, max_tokens=700, bits=4)
    P, n_pages = 32, 40
    held = {s: [] for s in range(7)}
    length = {s: 0 for s in range(7)}

    def free(h):
        return n_pages - len({id(p) for l in h.values() for p in l})

    done = 0
    for _ in range(800):
        op = r.choice(["extend", "reorder", "reorder", "truncate", "compact"])
        if op == "extend":
            seqs = r.sample(range(7), r.randint(0, 5))
            counts = [r.choice([0, 1, 1, 33, 70]) for _ in seqs]
            h2 = {s: list(l) for s, l in held.items()}
            for s, k in zip(seqs, counts):
                if k and length[s] % P and sum(any(x is h2[s][-1] for x in l) for l in h2.values()) > 1:
                    h2[s][-1] = object()
                h2[s] += [object() for _ in range(-(-(length[s] + k) // P) - len(h2[s]))]
            if free(h2) >= 0 and all(length[s] + k <= 400 for s, k in zip(seqs, counts)):
                c.extend(seqs, counts)
                held = h2
                for s, k in zip(seqs, counts):
                    length[s] += k
            else:
                refused(binding.E_CAPACITY, c.extend, seqs, counts)
        elif op == "reorder":
            seqs = r.sample(range(7), r.randint(0, 7))
            src = [r.randrange(7) for _ in seqs]
            c.reorder(seqs, src)
            h2, l2 = dict(held), dict(length)
            for s, f in zip(seqs, src):
                held[s], length[s] = list(h2[f]), l2[f]
            done += len(seqs)
        elif op == "truncate":
            seqs = r.sample(range(7), r.randint(0, 2))
            to = [r.choice([0, length[s] // 2, length[s]]) for s in seqs]
            c.truncate(seqs, to)
            for s, k in zip(seqs, to):
                length[s], held[s] = k, held[s][: -(-k // P)]
        else:
            c.compact()
        for s in range(7):
            assert c.info(s) == (length[s], len(held[s]), free(held))
    assert done > 500
