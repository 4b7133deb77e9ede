"""Device code of the operators around the FFN, compiled here for gfx950: what the
accesses assume about addresses.  CPU only."""
import os
import re
import subprocess

import pytest

from paper_2605_03667_amd import build

pytestmark = [pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="ROCm toolchain absent"), pytest.mark.slow]


def _device_ir(source, tmp_path):
    """(LLVM IR, diagnostics) of a source's device side with the build's flags."""
    out = str(tmp_path / "device.ll")
    r = subprocess.run(["/opt/rocm/bin/hipcc", *build.FLAGS, "--cuda-device-only", "-S", "-emit-llvm",
                        os.path.join(build.CSRC, source), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return open(out).read(), r.stderr


def test_gradient_tensors_need_their_elements_alignment_only(tmp_path):
    """The 16-byte accesses to gradients say so: 4 bytes for float32, 2 for bf16."""
    ir, messages = _device_ir("grad_clip.hip", tmp_path)
    assert "-Walign-mismatch" not in messages
    found = re.findall(r"(?:load|store) (<4 x float>|<4 x i32>)[^\n]* align (\d+)", ir)
    assert {(t, int(n)) for t, n in found} == {("<4 x float>", 4), ("<4 x i32>", 2)}
