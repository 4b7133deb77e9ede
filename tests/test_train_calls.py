"""What the entry points of include/elas_train.h hand on to their launch sequences:
the ABI layer compiled with launch sequences that only record their arguments; and
workspaces, their sizes and the device they must be on.  CPU only."""
import os
import subprocess

import pytest
import torch

import paper_2605_03667_amd as elas
from paper_2605_03667_amd import build, train

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"


@pytest.mark.slow
@pytest.mark.skipif(not os.path.exists(HIPCC), reason="ROCm toolchain absent")
def test_arguments_handed_on(tmp_path):
    objs = []
    for src in (os.path.join(build.CSRC, "train_api.hip"), os.path.join(ROOT, "tests", "sanitize", "train_calls.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", *build.FLAGS, "-O1", "-c", src, "-o", objs[-1]], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
    exe = str(tmp_path / "train_calls")
    r = subprocess.run([HIPCC, *objs, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "train calls: 0 failures" in r.stdout, r.stdout + r.stderr


class _OnDevice(torch.Tensor):
    """Bytes that call themselves a tensor on GPU 1."""

    def get_device(self):
        return 1


def test_workspace_on_the_operands_device():
    ws = torch.zeros(64, dtype=torch.uint8).as_subclass(_OnDevice)
    assert train._scratch(ws, 64, torch.device("cuda", 1))[2] == 64
    with pytest.raises(ValueError, match="workspace must be a GPU tensor on device 0"):
        train._scratch(ws, 64, torch.device("cuda", 0))


@pytest.mark.skipif(not os.path.exists(elas.LIB_PATH), reason="libelas.so not built")
def test_workspace_of_sizes_out_of_range():
    """No call takes these sizes; planning for them would leave the range of its integers."""
    big = 2 ** 63 - 1
    for T, d in ((big, 16), (1 << 31, 16), (4, big - 7), (4, 65544), (-1, 16), (4, 0)):
        assert elas.elas_norm_join_bwd_workspace_bytes(T, d) == 0
        for V in (10, 32000):
            assert elas.elas_embed_bwd_workspace_bytes(T, V, d) == 0
    for V in (big, 1 << 31, 0, -1):
        assert elas.elas_embed_bwd_workspace_bytes(5000, V, 16) == 0
    for n in (big, 1 << 20, -1):
        assert elas.elas_grad_workspace_bytes(n) == 0
    # the largest that are taken
    assert elas.elas_norm_join_bwd_workspace_bytes((1 << 31) - 1, 65536) > 0
    assert elas.elas_embed_bwd_workspace_bytes((1 << 31) - 1, (1 << 31) - 1, 65536) > 0
    assert elas.elas_grad_workspace_bytes((1 << 20) - 1) > 0


@pytest.mark.skipif(not os.path.exists(elas.LIB_PATH), reason="libelas.so not built")
def test_sort_workspace_does_not_grow_with_the_square():
    """Every workgroup of the sort reads all workgroups' counts (up to 2 KB each), so the
    counts may not grow with the tokens: beside 16 bytes a token there are those and the
    open sums of about 8192 chunks."""
    for T in (1 << 22, 1 << 26, (1 << 31) - 1):
        for V in (100, 32000, 1 << 27):
            for flags in (0, elas.ELAS_EMBED_ADD):
                assert elas.elas_embed_bwd_workspace_bytes(T, V, 8, flags) - 16 * T <= (1 << 20) + 9000 * 9 * 4 + 4096


@pytest.mark.skipif(not os.path.exists(elas.LIB_PATH), reason="libelas.so not built")
def test_norm_join_workgroups_fill_the_card_evenly():
    """The backward's workgroups, one row of sums in the workspace each: a whole number of them
    to each of the 256 CUs where there are rows for that."""
    for d in (8, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 6144, 8192, 8200, 65536):
        rows, rest = divmod(elas.elas_norm_join_bwd_workspace_bytes(1 << 20, d), 2 * d * 4)
        assert rest == 0 and rows % 256 == 0, d
