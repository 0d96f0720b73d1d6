"""What ps_soft reserves, on the host: tests/soft_plan_main.cpp builds the plans of csrc/soft_plan.h with the
undefined-behaviour sanitizer and compares reserved rooms with those of seeded smaller calls.  No GPU is involved."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


# products that the one folds before its sanitizer sees them, the other checks
@pytest.mark.parametrize("compiler", ["g++", "/opt/rocm/llvm/bin/clang++"])
def test_reserved_room_holds_every_smaller_call(tmp_path, compiler):
    if shutil.which(compiler) is None:
        pytest.skip(f"needs {compiler}")
    exe = str(tmp_path / "soft_plan")
    subprocess.run([compiler, "-std=c++17", "-O1", "-g", "-Wall", "-Wextra", "-Werror", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", os.path.join(HERE, "soft_plan_main.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, env=dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1"), timeout=300)
    assert r.returncode == 0, (r.stdout[-4000:], r.stderr[-4000:])
    assert "0 failures" in r.stdout
