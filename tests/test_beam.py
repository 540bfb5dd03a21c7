"""Refusals of the beam selection's calls, on a handle without a device, and its
oracle against brute force (no GPU needed)."""
import math
import os

import numpy as np
import pytest

from oracle import operators as O
from paper_2507_01021_amd import binding

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH), reason="library not built")


def refused(status, f, *a, **kw):
    with pytest.raises(binding.WhisperError) as e:
        f(*a, **kw)
    assert e.value.status == status, e.value
    assert str(e.value)


@pytest.mark.parametrize("vocab,rows,device", [(0, 1, -1), ((1 << 20) + 1, 1, -1), (10, 0, -1), (10, 65537, -1), (10, 1, -2)])
def test_create_refuses(vocab, rows, device):
    refused(binding.E_DEVICE if device == -2 else binding.E_INVAL, binding.Beam, vocab, rows, device)


@pytest.mark.parametrize("suppress", [[33], [-1], list(range(33)), [2**40], [0.5]])
def test_options_refuse(suppress):
    b = binding.Beam(33, 4, binding.NO_DEVICE)
    b.options([0, 32, 0])
    refused(binding.E_INVAL, b.options, suppress)


def test_run_checks_its_arguments_first():
    b = binding.Beam(33, 20, binding.NO_DEVICE)
    ok = 4096

    def run(logits=ok, dtype=0, n_groups=2, width=5, n_best=10, scores=ok, parents=ok, tokens=ok, out=ok, row_stride=0):
        b.run(logits, dtype, n_groups, width, n_best, scores, parents, tokens, out, row_stride)

    for kw in (dict(dtype=2), dict(width=0), dict(width=33, n_groups=0), dict(n_best=0), dict(n_best=65), dict(n_groups=5),
               dict(n_groups=-1), dict(n_groups=4, width=6), dict(row_stride=32), dict(row_stride=-33),
               dict(row_stride=2**41), dict(logits=0), dict(scores=0), dict(parents=0), dict(tokens=0), dict(out=0),
               dict(logits=ok + 2), dict(logits=ok + 1, dtype=1), dict(scores=ok + 2), dict(parents=ok + 1),
               dict(tokens=ok + 2), dict(out=ok + 3)):
        refused(binding.E_INVAL, run, **kw)
    run(0, 0, 0, 5, 10, 0, 0, 0, 0)  # no groups
    refused(binding.E_STATE, run, logits=ok + 2, dtype=1)  # no device


def test_null_handles_are_refused():
    lib = binding.load()
    assert lib.whisper_beam_create(10, 1, -1, None) == binding.E_INVAL
    assert lib.whisper_beam_set_stream(None, None) == binding.E_INVAL
    assert lib.whisper_beam_options(None, None, 0) == binding.E_INVAL
    assert lib.whisper_beam_run(None, None, 0, 0, 1, 1, 0, None, None, None, None) == binding.E_INVAL
    lib.whisper_beam_destroy(None)
    b = binding.Beam(10, 1, binding.NO_DEVICE)
    assert lib.whisper_beam_options(b.h, None, 1) == binding.E_INVAL
    assert lib.whisper_beam_options(b.h, None, -1) == binding.E_INVAL
    assert b"suppress" in lib.whisper_beam_error(b.h)


def test_oracle_against_brute_force():
    r = np.random.default_rng(0)
    for width, ids, n in ((1, 1, 2), (3, 7, 5), (2, 4, 20), (4, 11, 9)):
        scores = -r.random(width) * 5
        logits = r.integers(-3, 3, (width, ids)).astype(float)  # ties
        if width > 2:
            scores[1] = -math.inf
            logits[2, 3] = math.nan
        suppress = [0] if ids > 4 else []
        every = []
        for b in range(width):
            left = [i for i in range(ids) if i not in suppress and not math.isnan(logits[b, i])]
            lse = math.log(sum(math.exp(logits[b, i]) for i in left))
            every += [(-(scores[b] + logits[b, i] - lse), b, i) for i in left if math.isfinite(scores[b])]
        # (equal ones to the last bit: round so that both sides order them alike)
        every.sort(key=lambda e: (round(e[0], 9), e[1], e[2]))
        p, t, s = O.continuations(scores, logits, n, suppress)
        m = min(n, len(every))
        assert [(b, i) for _, b, i in every[:m]] == list(zip(p[:m], t[:m]))
        assert np.allclose([-e[0] for e in every[:m]], s[:m], atol=1e-12)
        assert (p[m:] == -1).all() and (t[m:] == -1).all() and (s[m:] == -math.inf).all()
