"""Refusals of the sampler's calls, on a handle without a device (no GPU needed)."""
import ctypes as C
import os

import pytest

from paper_2507_01021_amd import binding

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH), reason="library not built")


def refused(status, f, *a, **kw):
    with pytest.raises(binding.WhisperError) as e:
        f(*a, **kw)
    assert e.value.status == status, e.value
    assert str(e.value)


@pytest.mark.parametrize("vocab,rows,device", [(0, 1, -1), ((1 << 20) + 1, 1, -1), (10, 0, -1), (10, 65537, -1), (10, 1, -2)])
def test_create_refuses(vocab, rows, device):
    refused(binding.E_DEVICE if device == -2 else binding.E_INVAL, binding.Sampler, vocab, rows, device)


@pytest.mark.parametrize("kw", [
    dict(temperature=-0.1), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_k=-1),
    dict(top_k=1.5), dict(top_k=2**31), dict(top_p=0.0), dict(top_p=1.001), dict(top_p=float("nan")), dict(min_p=-0.1),
    dict(min_p=1.1), dict(min_p=float("nan")), dict(temperature=[1.0, 1.0]), dict(suppress=[33]), dict(suppress=[-1]),
    dict(suppress=list(range(33))), dict(n_rows=5), dict(suppress=[2**40])])
def test_options_refuse(kw):
    s = binding.Sampler(33, 4, binding.NO_DEVICE)
    s.options(temperature=[0.0, 0.5, 1.0, 2.0], top_k=[0, 1, 33, 2**31 - 1], top_p=[1.0, 1e-9, 0.5, 0.9], min_p=0.1,
              suppress=[0, 32, 0])
    refused(binding.E_INVAL, s.options, **(dict(n_rows=4) | kw))


def test_run_checks_its_arguments_first():
    s = binding.Sampler(33, 4, binding.NO_DEVICE)
    ok = 4096
    refused(binding.E_INVAL, s.run, ok, 2, 1, ok, ok)
    refused(binding.E_INVAL, s.run, ok, 0, 5, ok, ok)
    refused(binding.E_INVAL, s.run, ok, 0, -1, ok, ok)
    refused(binding.E_INVAL, s.run, ok, 0, 1, ok, ok, 0, 32)
    refused(binding.E_INVAL, s.run, 0, 0, 1, ok, ok)
    refused(binding.E_INVAL, s.run, ok, 0, 1, 0, ok)
    refused(binding.E_INVAL, s.run, ok, 0, 1, ok, 0)
    refused(binding.E_INVAL, s.run, ok + 2, 0, 1, ok, ok)
    refused(binding.E_INVAL, s.run, ok, 1, 1, ok + 1, ok)
    refused(binding.E_INVAL, s.run, ok, 1, 1, ok, ok, ok + 2)
    s.run(0, 0, 0, 0, 0)  # no rows
    refused(binding.E_STATE, s.run, ok + 2, 1, 1, ok, ok)  # no device


def test_null_handles_are_refused():
    lib = binding.load()
    assert lib.whisper_sampler_create(10, 1, -1, None) == binding.E_INVAL
    assert lib.whisper_sampler_set_stream(None, None) == binding.E_INVAL
    assert lib.whisper_sampler_options(None, None, 0, None, 0) == binding.E_INVAL
    assert lib.whisper_sampler_run(None, None, 0, 0, 0, None, None, None) == binding.E_INVAL
    lib.whisper_sampler_destroy(None)
    s = binding.Sampler(10, 1, binding.NO_DEVICE)
    assert lib.whisper_sampler_options(s.h, None, 1, None, 0) == binding.E_INVAL
    assert lib.whisper_sampler_options(s.h, None, 0, None, 1) == binding.E_INVAL


def test_sampling_layout_matches_header(tmp_path):
    import subprocess
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "whisper_mi355x.h")
    src = tmp_path / "layout.c"
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{header}"', "int main(void) {"]
    classes = {"whisper_sampling": binding.whisper_sampling, "whisper_cache_params": binding.whisper_cache_params}
    for st, cls in classes.items():
        lines.append(f'printf("%zu\\n", sizeof({st}));')
        lines += [f'printf("%zu\\n", offsetof({st}, {f}));' for f, _ in cls._fields_]
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-o", str(tmp_path / "layout"), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True,
                                          check=True).stdout.split()]
    want = []
    for cls in classes.values():
        want += [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want
