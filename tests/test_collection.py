"""GPU tests and Python's cyclic collector. `with pytest.raises(...) as e` in a
test's own frame makes a cycle (frame, e, traceback, frame), so what that test
holds, recorded graphs and handles among it, lives on until the collector runs. It
must not run while another test records: a graph that is destroyed then
synchronises the device, which a recording forbids, and its destructor ends the
process. (No GPU needed: the tests in TESTS hold plain objects.)"""
import os
import shutil
import subprocess
import sys

TESTS = '''
import gc
import weakref

import pytest

gc.set_threshold(10 ** 6)  # the collector happens not to run between tests
kept = []


class Graph:
    pass


def refused(f):
    with pytest.raises(ValueError) as e:
        f()
    assert e.value.args


@pytest.mark.gpu
@pytest.mark.parametrize("helper", [False, True])
def test_refuses(helper):
    assert not any(r() for r in kept)  # what earlier tests held is gone
    graph = Graph()
    kept.append(weakref.ref(graph))
    if helper:
        refused(lambda: int("x"))
    else:
        with pytest.raises(ValueError) as e:
            int("x")
        assert e.value.args


@pytest.mark.gpu
def test_records():
    assert len(kept) == 2 and not any(r() for r in kept)
    assert not gc.isenabled()  # nor does anything go while a test runs


def test_without_a_gpu():
    assert gc.isenabled()
'''


def test_nothing_is_collected_while_a_gpu_test_records(tmp_path):
    shutil.copy(os.path.join(os.path.dirname(os.path.abspath(__file__)), "conftest.py"), tmp_path)
    (tmp_path / "test_inner.py").write_text(TESTS)
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "--rootdir", str(tmp_path), str(tmp_path)],
                       capture_output=True, text=True, timeout=120, cwd=tmp_path)
    assert r.returncode == 0 and "4 passed" in r.stdout, r.stdout[-3000:]
