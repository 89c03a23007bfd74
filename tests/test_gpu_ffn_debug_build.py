"""The feed-forward operators on the debug library (-DSADMM_DEBUG, loaded when SADMM_DEBUG=1):
their kernels' loads and stores check their index too, and the parity suites, which
read the status word, stay clear.  In a child process, since a process loads one
library.  (That a check is there cannot be shown from outside: these kernels take no
index from memory that a test could spoil.)"""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TESTS = os.path.join(ROOT, "tests")
CSRC = os.path.join(ROOT, "paper_1807_11091_gb300", "csrc")


@pytest.mark.parametrize("name", ["norm.cu", "linear.cu", "few.cu", "output.cuh", "tgemm_dev.cuh"])
def test_the_sources_check_their_indexes(name):
    """Each of a source's 16-byte loads, bulk copies and row stores stands beside a check."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    checks = len(re.findall(r"\bdbg_(?:in|run)\(", text))
    assert checks >= {"norm.cu": 4, "linear.cu": 7, "few.cu": 3, "output.cuh": 2, "tgemm_dev.cuh": 8}[name]


@pytest.mark.gpu
def test_parity_suites_pass_on_the_debug_library():
    env = dict(os.environ)
    env["SADMM_DEBUG"] = "1"
    env["PYTHONPATH"] = os.pathsep.join([ROOT, TESTS, env.get("PYTHONPATH", "")])
    which = ("from paper_1807_11091_gb300 import sadmm; sadmm.load(); "
             "assert sadmm.library_path().endswith('debug/libsadmm.so'), sadmm.library_path()")
    r = subprocess.run([sys.executable, "-c", which], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    files = ["test_gpu_layernorm.py", "test_gpu_linear.py", "test_gpu_ffn_block.py", "test_gpu_ffn_small_blocks.py",
             "test_gpu_ffn_long_sums.py", "test_gpu_ffn_activations.py"]
    cmd = [sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider"]
    cmd += [os.path.join(TESTS, f) for f in files]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=1800)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
