"""The adapters' tests under the checked build of the library (-DRABIT_CHECKED): every address that their kernels make from ids, lists of rows and sizes is compared with
its buffer, reads as well as writes.  They must pass, and no check may have failed.  The checked library is a separate file, selected through RABIT_LIBRARY, so this runs in
a child process."""
import importlib.util
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import sys
import pytest
code = pytest.main(["-x", "-q", "-m", "gpu", "-p", "no:cacheprovider"] + sys.argv[1:])
from paper_2602_05367_b200 import binding
faults = binding.raw_lib().rabit_selftest_index_faults()
print("index faults:", faults, binding.last_error())
sys.exit(int(code) or int(faults != 0))
"""


@pytest.mark.gpu
def test_the_adapters_pass_under_the_checked_build():
    spec = importlib.util.spec_from_file_location("_rabit_build", os.path.join(ROOT, "paper_2602_05367_b200", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    lib = build.LIB_CHECKED
    sources = [os.path.join(build.CSRC, f) for f in os.listdir(build.CSRC)]
    if not os.path.exists(lib) or any(os.path.getmtime(f) > os.path.getmtime(lib) for f in sources):
        build.build(checked=True)
    cmd = [sys.executable, "-c", CHILD, os.path.join(ROOT, "tests", "test_gpu_adapters.py"), os.path.join(ROOT, "tests", "test_gpu_adapters_calls.py"),
           "-k", "adapted or finite or any_size or chain or captured or gradients or training or 32_bits or slot or small_low_rank or narrow_sides"]
    proc = subprocess.run(cmd, cwd=ROOT, env=dict(os.environ, RABIT_LIBRARY=lib), capture_output=True, text=True, timeout=1200)
    assert proc.returncode == 0, proc.stdout[-3000:] + proc.stderr[-2000:]
    assert " passed" in proc.stdout and "index faults: 0" in proc.stdout


def test_the_ordinary_build_has_no_checks():
    from paper_2602_05367_b200 import binding
    if os.environ.get("RABIT_LIBRARY"):
        pytest.skip("another library is loaded")
    assert binding.raw_lib().rabit_selftest_index_faults() == -2 and "RABIT_CHECKED" in binding.last_error()
