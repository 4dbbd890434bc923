"""The compiler's own check of the machine code of the kernels around the bounded cache.

One of its passes loses live ranges of 16-byte loads whose words are used one by one (the
attention sources are built without it); outputs are wrong then, with no error, and
only on the paths that the pass has touched.  The verifier names such a range."""
import concurrent.futures as cf
import os
import signal
import subprocess

import pytest

from paper_2606_24467_amd import build as B

SOURCES = ["attend_fp4.hip", "attend_bf16.hip", "attend_f32.hip", "attend.hip", "window_prompt.hip",
           "cache.hip"]


def _verify(src, out):
    """Exit code and messages of a device compilation with the verifier on."""
    cmd = [B._hipcc(), *B.FLAGS, *B.EXTRA.get(src, []), "-mllvm", "-verify-machineinstrs",
           "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", str(out / (src + ".s"))]
    log = out / (src + ".log")
    with open(log, "wb") as f:
        p = subprocess.Popen(cmd, stdin=subprocess.DEVNULL, stdout=f, stderr=f,
                             start_new_session=True)
        try:
            code = p.wait(timeout=400)
        except subprocess.TimeoutExpired:
            os.killpg(p.pid, signal.SIGKILL)
            code = p.wait()
    return code, log.read_text(errors="replace")


@pytest.fixture(scope="module")
def verified(tmp_path_factory):
    out = tmp_path_factory.mktemp("codegen")
    with cf.ThreadPoolExecutor(len(SOURCES)) as pool:
        return dict(zip(SOURCES, pool.map(lambda s: _verify(s, out), SOURCES)))


@pytest.mark.parametrize("src", SOURCES)
def test_machine_code_passes_the_verifier(verified, src):
    code, log = verified[src]
    assert "Bad machine code" not in log, log[:2000]
    assert code == 0, log[:2000]
