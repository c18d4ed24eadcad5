"""The checks and plans of user histories under the host sanitizers, as tests/test_sanitizers.py has those of the forward pass.  No device."""
import os
import sys

import pytest

from test_sanitizers import _preload, _run


def test_history_host_code_under_address_and_ub_sanitizers():
    from paper_2203_07424_amd import build
    lib, runtime = build.build_host_sanitized(), build.sanitizer_runtime()
    if not os.path.isabs(runtime) or not os.path.exists(runtime):
        pytest.skip("no clang AddressSanitizer runtime here")
    env = _preload(dict(os.environ), runtime)
    env["REC_MI355X_LIBRARY"] = lib
    out = _run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_history_refusals.py",
                "tests/test_history_host.py", "tests/test_history_forms.py"], env)
    assert " passed" in out and "failed" not in out, out[-2000:]
