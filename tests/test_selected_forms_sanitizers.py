"""The choice of forms of tests/test_selected_forms.py under the host sanitizers.  No device."""
import os
import sys

import pytest

from test_sanitizers import _preload, _run


def test_forms_under_address_and_ub_sanitizers():
    from paper_2203_07424_amd import build
    lib, runtime = build.build_host_sanitized(), build.sanitizer_runtime()
    if not os.path.isabs(runtime) or not os.path.exists(runtime):
        pytest.skip("no clang AddressSanitizer runtime here")
    env = _preload(dict(os.environ), runtime)
    env["REC_MI355X_LIBRARY"] = lib
    out = _run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_selected_forms.py"], env)
    assert " passed" in out and "failed" not in out, out[-2000:]
