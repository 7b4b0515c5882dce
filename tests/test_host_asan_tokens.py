"""The host code of the operators for drafted trees and for eviction under AddressSanitizer (CPU only): their refusals, the checks
of overlapping rows and the planners' workspaces (test_abi_tokens.py) against the library whose host pass is instrumented, in a
child process that preloads the sanitizer's runtime."""
import os
import subprocess
import sys

import pytest

from paper_2608_02691_amd import build as B

from test_host_asan import ROOT, _stale

_CHILD = r"""
import ctypes, itertools, sys
sys.path.insert(0, {root!r}); sys.path.insert(0, {tests!r})
assert hasattr(ctypes.CDLL(None), "__asan_init"), "sanitizer runtime not loaded"
from paper_2608_02691_amd import int2kv as K
lib = K.load_library({lib!r})
import test_abi_tokens
calls = 0
for module in (test_abi_tokens,):
    for name in sorted(n for n in dir(module) if n.startswith("test_")):
        test, choices = getattr(module, name), []
        for mark in getattr(test, "pytestmark", []):
            names = [x.strip() for x in mark.args[0].split(",")]
            choices.append([dict(zip(names, v if len(names) > 1 else (v,))) for v in mark.args[1]])
        for choice in itertools.product(*choices):
            test(**{{k: v for c in choice for k, v in c.items()}})
            calls += 1
print("host checks under the sanitizer:", calls, flush=True)
assert calls > 70
"""


def test_host_code_of_trees_and_eviction_is_clean_under_address_sanitizer():
    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc is not installed")
    rt = B.asan_runtime()
    if not rt:
        pytest.skip("the compiler's shared AddressSanitizer runtime is not installed")
    if _stale(B.ASAN_LIB):
        B.build_host_asan()
    env = dict(os.environ)
    env["LD_PRELOAD"] = " ".join(p for p in (rt, os.environ.get("LD_PRELOAD", "")) if p)
    env["ASAN_OPTIONS"] = "detect_leaks=0:halt_on_error=1:verify_asan_link_order=0"
    code = _CHILD.format(root=ROOT, tests=os.path.join(ROOT, "tests"), lib=B.ASAN_LIB)
    r = subprocess.run([sys.executable, "-c", code], env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, timeout=600)
    out = r.stdout.decode(errors="replace")
    assert "AddressSanitizer" not in out, out[-4000:]
    assert r.returncode == 0 and "host checks under the sanitizer:" in out, out[-4000:]
