"""The paged cache's book and the refusals of its calls, on a handle without a
device (no GPU needed): lengths, shared pages, free pages, and that a refused
call changes nothing."""
import ctypes as C
import os
import random

import pytest

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


@pytest.mark.parametrize("field,value", [
    ("dtype", 2), ("n_layer", 0), ("n_layer", 257), ("n_head", 3), ("n_head", 0), ("n_kv_head", 0), ("n_head", 258),
    ("head_size", 80), ("page_size", 16), ("page_size", 48), ("n_pages", 0), ("max_seqs", 0), ("max_seqs", 4097),
    ("max_positions", 0), ("max_tokens", 0), ("max_tokens", (1 << 20) + 1), ("device", -2)])
def test_create_refuses(field, value):
    refused(binding.E_DEVICE if field == "device" else binding.E_INVAL, cache, **{field: value})


def test_null_handles_are_refused():
    lib = binding.load()
    i = C.c_int32()
    assert lib.whisper_cache_create(None, 0, None) == binding.E_INVAL
    assert lib.whisper_cache_set_stream(None, None) == binding.E_INVAL
    assert lib.whisper_cache_extend(None, None, None, 0) == binding.E_INVAL
    assert lib.whisper_cache_append(None, 0, None, None, 0, 0) == binding.E_INVAL
    assert lib.whisper_cache_attend(None, 0, None, None, 0, 0, 1.0) == binding.E_INVAL
    assert lib.whisper_cache_truncate(None, None, None, 0) == binding.E_INVAL
    assert lib.whisper_cache_fork(None, 0, None, 0) == binding.E_INVAL
    assert lib.whisper_cache_compact(None) == binding.E_INVAL
    assert lib.whisper_cache_read(None, 0, None, 0, None, None, 0, 0) == binding.E_INVAL
    assert lib.whisper_cache_info(None, 0, C.byref(i), None, None) == binding.E_INVAL
    lib.whisper_cache_destroy(None)


def test_lists_are_checked():
    c = cache()
    c.extend([0], [40])
    refused(binding.E_CAPACITY, c.extend, [6], [1])
    refused(binding.E_CAPACITY, c.extend, [-1], [1])
    refused(binding.E_INVAL, c.extend, [1, 1], [1, 1])
    refused(binding.E_INVAL, c.extend, [1], [-1])
    refused(binding.E_INVAL, c.extend, [1, 2], [1])
    refused(binding.E_INVAL, c.extend, [2**31], [1])
    refused(binding.E_INVAL, c.truncate, [0], [41])
    refused(binding.E_INVAL, c.truncate, [0], [-1])
    refused(binding.E_INVAL, c.truncate, [0, 0], [1, 1])
    refused(binding.E_CAPACITY, c.truncate, [9], [0])
    refused(binding.E_INVAL, c.fork, 0, [0])
    refused(binding.E_INVAL, c.fork, 0, [1, 1])
    refused(binding.E_CAPACITY, c.fork, 6, [1])
    refused(binding.E_CAPACITY, c.fork, 0, [6])
    refused(binding.E_STATE, c.fork, 1, [0])
    assert [c.info(s)[0] for s in range(6)] == [40, 0, 0, 0, 0, 0] and c.info(0)[1:] == (2, 6)


def test_device_calls_check_their_arguments_first():
    c = cache()
    c.extend([0], [1])
    ok = 4096
    for layer in (-2, 2):
        refused(binding.E_INVAL, c.append, layer, ok, ok)
        refused(binding.E_INVAL, c.read, layer, [0], ok, ok)
    for layer in (-1, 2):
        refused(binding.E_INVAL, c.attend, layer, ok, ok)
    refused(binding.E_INVAL, c.append, 0, 0, ok)
    refused(binding.E_INVAL, c.append, 0, ok, ok + 1)
    refused(binding.E_INVAL, c.append, 0, ok, ok, k_stride=127)
    refused(binding.E_INVAL, c.append, 0, ok, ok, v_stride=-128)
    refused(binding.E_INVAL, c.attend, 0, ok + 2, ok)
    refused(binding.E_INVAL, c.attend, 0, ok, ok + 8)
    refused(binding.E_INVAL, c.attend, 0, ok, ok, q_stride=260)
    refused(binding.E_INVAL, c.attend, 0, ok, ok, out_stride=255)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refused(binding.E_INVAL, c.attend, 0, ok, ok, scale=scale)
    refused(binding.E_STATE, c.append, 0, ok, ok)  # no device
    refused(binding.E_STATE, c.attend, 0, ok, ok)
    refused(binding.E_STATE, c.read, 0, [0], ok, ok)
    refused(binding.E_CAPACITY, c.read, 0, [7], ok, ok)


def test_capacity_is_checked_before_anything_changes():
    c = cache()
    c.extend([0, 1], [100, 64])  # 4 + 2 pages
    assert c.info(0)[2] == 2
    refused(binding.E_CAPACITY, c.extend, [2, 0], [32, 61])  # 1 + 2 pages, 2 free
    refused(binding.E_CAPACITY, c.extend, [0], [101])  # max_positions
    refused(binding.E_CAPACITY, c.extend, [0, 1, 2], [100, 100, 101])  # max_tokens
    assert [c.info(s) for s in (0, 1, 2)] == [(100, 4, 2), (64, 2, 2), (0, 0, 2)]
    refused(binding.E_CAPACITY, c.fork, 0, [2, 3, 4])  # three copies of a partial page
    assert c.info(2) == (0, 0, 2)
    c.fork(1, [2, 3, 4])  # whole pages only: nothing is needed
    assert c.info(4) == (64, 2, 2)


def test_shared_pages_are_copied_when_written():
    c = cache()
    c.extend([0], [70])  # 3 pages
    c.fork(0, [1])       # 2 shared, 1 copied
    assert c.info(1) == (70, 3, 4)
    c.truncate([0, 1], [50, 50])  # the second page is now partly used, and shared
    assert c.info(0) == (50, 2, 6)
    c.extend([0, 1], [1, 1])  # the first writer gets a copy, the last one writes in place
    assert c.info(0)[2] == 5
    c.truncate([0], [0])
    assert c.info(1) == (51, 2, 6)
    c.truncate([1], [0])
    assert c.info(1) == (0, 0, 8)


def test_sequences_of_one_call_that_share_their_last_page():
    c = cache(n_pages=4)
    c.extend([0], [64])
    c.fork(0, [1, 2])
    c.truncate([0, 1, 2], [40, 40, 40])  # all three in one shared page, 2 pages free
    c.extend([0, 1, 2], [1, 0, 1])       # 0 is copied, 2 is copied, 1 keeps it
    assert c.info(1) == (40, 2, 0)
    refused(binding.E_CAPACITY, c.fork, 0, [3])
    c.truncate([1], [0])
    assert c.info(1) == (0, 0, 1)


def test_random_calls_against_a_plain_book():
    r = random.Random(5)
    c = cache(n_pages=40, max_seqs=7, max_positions=400, max_tokens=500)
    P, n_pages = 32, 40
    held = {s: [] for s in range(7)}  # sequence -> page tokens; shared pages are the same object
    length = {s: 0 for s in range(7)}

    def free():
        return n_pages - len({id(p) for l in held.values() for p in l})

    done = 0
    for _ in range(600):
        op = r.choice(["extend", "extend", "truncate", "fork", "compact"])
        if op == "extend":
            seqs = r.sample(range(7), r.randint(0, 4))
            counts = [r.choice([0, 1, 5, 33, 90]) for _ in seqs]
            h2 = {s: list(l) for s, l in held.items()}
            for s, k in zip(seqs, counts):
                if k and length[s] % P:
                    if sum(any(x is h2[s][-1] for x in l) for l in h2.values()) > 1:
                        h2[s][-1] = object()
                h2[s] += [object() for _ in range(-(-(length[s] + k) // P) - len(h2[s]))]
            fits = len({id(p) for l in h2.values() for p in l}) <= n_pages and all(
                length[s] + k <= 400 for s, k in zip(seqs, counts))
            if fits:
                c.extend(seqs, counts)
                held = h2
                for s, k in zip(seqs, counts):
                    length[s] += k
                done += 1
            else:
                refused(binding.E_CAPACITY, c.extend, seqs, counts)
        elif op == "truncate":
            seqs = r.sample(range(7), r.randint(0, 3))
            to = [r.choice([0, length[s] // 2, length[s]]) for s in seqs]
            c.truncate(seqs, to)
            for s, k in zip(seqs, to):
                length[s] = k
                held[s] = held[s][: -(-k // P)]
        elif op == "fork":
            src = r.randrange(7)
            dst = [s for s in range(7) if s != src and length[s] == 0][: r.randint(0, 3)]
            part = length[src] % P != 0
            if part and len(dst) > free():
                refused(binding.E_CAPACITY, c.fork, src, dst)
                continue
            c.fork(src, dst)
            for d in dst:
                held[d] = list(held[src])
                if part:
                    held[d][-1] = object()
                length[d] = length[src]
        else:
            c.compact()
        for s in range(7):
            assert c.info(s) == (length[s], len(held[s]), free())
    assert done > 50
