"""The operators with 8-bit operands on the debug library (-DSADMM_DEBUG, loaded when
SADMM_DEBUG=1): their kernels' loads and stores check their index too, and the parity
suites, which read the status word, stay clear.  In a child process, since a process
loads one library.  And what their waits must not stand behind."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TESTS = os.path.join(ROOT, "tests")
CSRC = os.path.join(ROOT, "paper_1807_11091_gb300", "csrc")


def code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


@pytest.mark.parametrize("name,least", [("rms.cu", 5), ("quant.cu", 6), ("linear8.cu", 2), ("q8gemm.cu", 2), ("q8pair.cu", 1)])
def test_the_sources_check_their_indexes(name, least):
    assert len(re.findall(r"\bdbg_(?:in|run)\(", code(name))) >= least


@pytest.mark.parametrize("name", ["q8pair.cu", "q8gemm.cu"])
def test_no_barrier_behind_a_wait_that_may_give_up(name):
    """Each warp finds out for itself that a wait gave up, so none may stand at a barrier without a limit
    before all have left their loops."""
    text = code(name)
    assert not re.search(r"\bbar(rier)?\.(cta\.)?(sync|red|arrive)|named_barrier", text)
    for line in text.split("\n"):
        if "__syncthreads()" in line or "cluster_sync()" in line:
            assert len(line) - len(line.lstrip()) == 4, line


@pytest.mark.gpu
def test_parity_suites_pass_on_the_debug_library():
    env = dict(os.environ)
    env["SADMM_DEBUG"] = "1"
    env["PYTHONPATH"] = os.pathsep.join([ROOT, TESTS, env.get("PYTHONPATH", "")])
    which = ("from paper_1807_11091_gb300 import sadmm; sadmm.load(); "
             "assert sadmm.library_path().endswith('debug/libsadmm.so'), sadmm.library_path()")
    r = subprocess.run([sys.executable, "-c", which], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    files = ["test_gpu_rmsnorm.py", "test_gpu_quantize.py", "test_gpu_linear8.py", "test_gpu_gated8.py", "test_gpu_ffn8_block.py"]
    cmd = [sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider"]
    cmd += [os.path.join(TESTS, f) for f in files]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=1800)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
