"""Device code of the losses and of AdamW, compiled here for gfx950: what the accesses assume about
addresses.  CPU only."""
import re

import pytest

from test_train_device_code import _device_ir, pytestmark  # noqa: F401


def _vectors(ir):
    """(type, alignment) of the vector loads and stores in global memory."""
    found = re.findall(r"(?:load|store) (<\d+ x (?:float|i32)>),? [^\n]*?align (\d+)", ir)
    found += re.findall(r"store (<\d+ x (?:float|i32)>) [^\n]* align (\d+)", ir)
    return {(t, int(n)) for t, n in found}


def test_logits_need_their_elements_alignment_only(tmp_path):
    """The 16-byte accesses to logits and gradients say so: 4 bytes for float32, 2 for bf16."""
    ir, messages = _device_ir("token_loss.hip", tmp_path)
    assert "-Walign-mismatch" not in messages
    assert {v for v in _vectors(ir) if v[0] in ("<4 x float>", "<4 x i32>")} == {("<4 x float>", 4), ("<4 x i32>", 2)}


@pytest.mark.parametrize("source", ["preference.hip", "adamw.hip"])
def test_values_need_their_elements_alignment_only(source, tmp_path):
    """16 bytes of float32 values, 8 of bf16; the moments' own accesses (16 bytes of float32) are aligned."""
    ir, messages = _device_ir(source, tmp_path)
    assert "-Walign-mismatch" not in messages
    seen = _vectors(ir)
    assert ("<4 x float>", 4) in seen
    if source == "adamw.hip":
        assert ("<2 x i32>", 2) in seen and ("<4 x float>", 16) in seen
    assert {v for v in seen if v[0] == "<4 x float>"} <= {("<4 x float>", 4), ("<4 x float>", 16)}
