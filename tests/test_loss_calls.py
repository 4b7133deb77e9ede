"""Which calls of include/elas_loss.h and include/elas_adamw.h are handed on to their launch sequences: the ABI layer
compiled with launch sequences that only count, under the host's undefined-behaviour sanitizer; and what the binding
makes of a refusal.  CPU only."""
import os
import subprocess

import pytest
import torch

import paper_2605_03667_amd as elas
from paper_2605_03667_amd import build
from paper_2605_03667_amd import loss as binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"


@pytest.mark.slow
@pytest.mark.skipif(not os.path.exists(HIPCC), reason="ROCm toolchain absent")
def test_results_that_overlap_are_refused(tmp_path):
    """Every result over every other buffer of its call, in whole or by a byte, and beside it."""
    san = ["-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    objs = []
    for src in (os.path.join(build.CSRC, "loss_api.hip"), os.path.join(build.CSRC, "adamw_api.hip"),
                os.path.join(ROOT, "tests", "sanitize", "loss_calls.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", *build.FLAGS, *san, "-O1", "-c", src, "-o", objs[-1]], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
    exe = str(tmp_path / "loss_calls")
    r = subprocess.run([HIPCC, *san, *objs, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "loss calls: 0 failures" in r.stdout, r.stdout + r.stderr[-3000:]


class _OnGpu(torch.Tensor):
    """Values that call themselves a tensor on GPU 0."""

    def get_device(self):
        return 0


@pytest.mark.skipif(not os.path.exists(elas.LIB_PATH), reason="libelas.so not built")
@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the tensors are not a GPU's")
def test_the_binding_raises_what_is_refused(monkeypatch):
    monkeypatch.setattr(binding, "_current", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda device: 0)
    gpu = lambda t: t.as_subclass(_OnGpu)  # noqa: E731
    rows, off = gpu(torch.zeros(64)), gpu(torch.arange(5))
    for out in ({"margin": rows[:2]}, {"dlogp": rows[32:48], "margin": rows[46:48]}):
        with pytest.raises(elas.ElasError, match="ELAS_ERR_OVERLAP: margin overlaps"):
            elas.elas_preference_loss(rows[:16], off, out={"stats": rows[60:63], **out})
    with pytest.raises(elas.ElasError, match="ELAS_ERR_OVERLAP: stats overlaps logp"):
        elas.elas_preference_loss(rows[:16], off, out={"stats": rows[13:16]})
