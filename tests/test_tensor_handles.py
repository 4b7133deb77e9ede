"""ElasTensors on the host: what it makes of torch's comparison of many tensors (an interface that another torch may
have changed), and what a handle costs whose tensors it cannot compare.  CPU only."""
import pytest
import torch

import paper_2605_03667_amd as elas
from paper_2605_03667_amd import train


class _OnGpu(torch.Tensor):
    """Values that call themselves a tensor on GPU 0."""

    def get_device(self):
        return 0


def _handle(*shapes):
    h = elas.ElasTensors([torch.zeros(s).as_subclass(_OnGpu) for s in shapes])
    h.device = torch.device("cuda", 0)
    return h


class _Guards:
    """Stands for torch's class: counts what is asked of it."""
    made = asked = 0
    answers = None      # one for each question; the last stays

    def __init__(self, *tensors, dynamic_dims_sizes=None, dynamic_dims_strides=None):
        type(self).made += 1

    def check(self, *tensors):
        cls = type(self)
        cls.asked += 1
        return cls.answers.pop(0) if len(cls.answers) > 1 else cls.answers[0]


def _guards(monkeypatch, answers):
    cls = type("Guards", (_Guards,), {"answers": list(answers)})
    monkeypatch.setattr(train, "TensorGuards", cls)
    return cls


@pytest.mark.parametrize("error", [TypeError, RuntimeError, AttributeError])
@pytest.mark.parametrize("where", ["__init__", "check"])
def test_a_torch_whose_guards_are_others(monkeypatch, where, error):
    """Any failure of the guards is as if there were none."""
    cls = _guards(monkeypatch, [True])

    def fails(self, *a, **k):
        raise error("another signature")

    monkeypatch.setattr(cls, where, fails)
    h = _handle(5, (2, 3))
    for _ in range(6):
        pointers, numel, types = h.arrays(written=True)
        assert list(numel) == [5, 6] and list(types) == [0, 0] and list(pointers) == [t.data_ptr() for t in h.tensors]
    h.tensors[0].data = torch.zeros(4, dtype=torch.bfloat16)
    assert list(h.arrays()[1]) == [4, 6]
    assert list(h.arrays()[2]) == [1, 0]


def test_a_guard_that_fails_once_it_is_in_use(monkeypatch):
    cls = _guards(monkeypatch, [True])
    h = _handle(5)
    for _ in range(3):
        h.arrays()

    def fails(self, *a):
        raise RuntimeError

    monkeypatch.setattr(cls, "check", fails)
    for _ in range(3):
        assert list(h.arrays()[1]) == [5]


@pytest.mark.parametrize("answers", [[False], [True, False], [True, True, True, False]])
def test_a_guard_that_says_no_to_what_has_not_changed(monkeypatch, answers):
    """It is asked a few times and then no more."""
    cls = _guards(monkeypatch, answers)
    h = _handle(5, 6)
    for _ in range(50):
        assert list(h.arrays()[1]) == [5, 6]
    assert cls.made <= 4 and cls.asked <= 12
    # tensors that did change are worth another
    made = cls.made
    h.tensors[1].data = torch.zeros(7)
    cls.answers[:] = [True]
    for _ in range(4):
        assert list(h.arrays()[1]) == [5, 7]
    assert cls.made > made


def test_a_guard_that_says_yes_stays(monkeypatch):
    cls = _guards(monkeypatch, [True])
    h = _handle(5)
    for _ in range(20):
        h.arrays()
    assert cls.made == 1 and 18 <= cls.asked <= 20


def test_torchs_own_guards():
    """With the installed torch: a tensor twice, and modes that differ from call to call."""
    t = torch.zeros(5).as_subclass(_OnGpu)
    h = elas.ElasTensors([t, t])
    h.device = torch.device("cuda", 0)
    for _ in range(6):
        assert list(h.arrays()[1]) == [5, 5]
    h = _handle(5, 6)
    for mode in (torch.enable_grad, torch.no_grad, torch.inference_mode) * 5:
        with mode():
            assert list(h.arrays()[1]) == [5, 6]
    h.tensors[0].data = torch.zeros(8)
    assert list(h.arrays()[1]) == [8, 6]
