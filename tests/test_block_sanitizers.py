"""The block cache calls' argument checks and planning under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only, as in
test_sanitizers.py): the host-only units rebuilt, their tests run again in a child process."""
import subprocess
import sys
from pathlib import Path

import pytest

from test_sanitizers import ROOT, _env, _report


def test_block_cache_host_code_under_address_and_ub_sanitizers(tmp_path):
    from paper_2506_19830_amd import build as hip_build
    try:
        rt = hip_build.asan_runtime()
    except FileNotFoundError:
        pytest.skip("hipcc's clang has no shared AddressSanitizer runtime here")
    lib = hip_build.build_host_sanitized(tmp_path / "libla_verify_san.so")
    check = ("import ctypes, sys; assert hasattr(ctypes.CDLL(None), '__asan_init'), 'sanitizer runtime not loaded'; "
             "from pathlib import Path; from paper_2506_19830_amd import binding as B; "
             f"B.LIB_PATH = Path({str(lib)!r}); "
             "import pytest; sys.exit(pytest.main(['-x', '-q', '-p', 'no:cacheprovider', 'tests/test_block_abi.py']))")
    r = subprocess.run([sys.executable, "-c", check], cwd=ROOT, env=_env(Path(rt)), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, _report(r)
    assert " passed" in r.stdout and "failed" not in r.stdout, _report(r)
