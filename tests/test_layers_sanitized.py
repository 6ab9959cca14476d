"""The host code of the operators between linear layers under the sanitizers of test_sanitizers.py (CPU only): what they
refuse, before any device call."""
import importlib.util
import os

import pytest

from test_sanitizers import ROOT, _clang_asan, _run_child


def test_refusals_under_asan_ubsan(tmp_path):
    rt = _clang_asan()
    if rt is None:
        pytest.skip("clang's ASan runtime is not installed")
    spec = importlib.util.spec_from_file_location("_galore_build_layers_san",
                                                  os.path.join(ROOT, "paper_2504_20437_amd", "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    mod.HIPCC_FLAGS = mod.HIPCC_FLAGS + ["-parallel-jobs=%d" % min(os.cpu_count() or 1, 8)]
    lib = mod.build_sanitized(str(tmp_path / "libgalore_san.so"))
    out = _run_child(["tests/test_layers_refusals.py", "tests/test_layers_limits.py"], {"GALORE_LIB": lib}, rt)
    assert "passed" in out
