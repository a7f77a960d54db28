"""The package without its extension module, or with one built for another torch: the calls that need it say so, all
others work."""
import os
import subprocess
import sys

import pytest

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# what stands in for the module: none, one built for another torch, one that does not say for what, the one that is there under a torch
# that lacks the private name of the raw stream
STANDINS = {
    "absent": "sys.modules['paper_2311_05161_b200._calls'] = None",
    "stale": "m = types.ModuleType('x'); m.built_for = 'torch 1.0, cpython-30'; m.set_errors = None; "
             "sys.modules['paper_2311_05161_b200._calls'] = m",
    "unmarked": "sys.modules['paper_2311_05161_b200._calls'] = types.ModuleType('x')",
    "no raw stream": "import torch; del torch._C._cuda_getCurrentRawStream",
}
PROGRAM = """
import sys, types
sys.path.insert(0, %r)
%s
import paper_2311_05161_b200 as w4a8
assert w4a8.packed_bytes(256, 256, 0) > 0 and w4a8.kv_page_bytes(16, 1, 64) == 16 * 72
assert len(w4a8.dint4_table(3)) == 16
try:
    w4a8.kv_append(None, None, None, None, None, None)
except ImportError as e:
    print("ImportError", e)
except TypeError as e:
    print("TypeError", e)
"""


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


@pytest.mark.parametrize("case", sorted(STANDINS))
def test_import(case):
    got = subprocess.run([sys.executable, "-c", PROGRAM % (ROOT, STANDINS[case])], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0, got.stderr[-2000:]
    if case == "no raw stream":
        assert got.stdout.startswith("TypeError K: expected a tensor")
    else:
        assert got.stdout.startswith("ImportError kv_append needs the extension module _calls")
        assert ("torch 1.0" in got.stdout) == (case == "stale")


def test_a_module_built_for_another_torch_is_stale(monkeypatch):
    assert not entry._calls_are_stale()
    monkeypatch.setattr(entry, "_calls_target", lambda: "torch 1.0, cpython-30")
    assert entry._calls_are_stale()
