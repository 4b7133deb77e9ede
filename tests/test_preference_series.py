"""The series of the preference loss's exponential and logarithm, evaluated from the source's coefficients over the range
that the kernel uses them in: as exact as the tests of its results allow for (2e-10 a sigmoid, of which
the exponential and the sum with it have half).  CPU only."""
import os
import re

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _series(name, x):
    text = open(os.path.join(ROOT, "paper_2605_03667_amd", "csrc", "preference.hip")).read()
    terms = re.search(name + r"\[(\d+)\] = \{(.*?)\}", text)
    values = [float(a) / float(b or 1) for a, b in re.findall(r"([0-9.]+)(?: / ([0-9.]+))?", terms.group(2))]
    assert len(values) == int(terms.group(1))
    return np.polyval(values, x)


def test_exponential():
    # (the rest of x less its nearest multiple of ln 2)
    x = np.linspace(-0.5 * np.log(2), 0.5 * np.log(2), 100001)
    assert np.abs(_series("kExpSeries", x) / np.exp(x) - 1).max() <= 1e-10


def test_logarithm():
    e = np.linspace(0, 1, 100001)[1:]
    s = e / (2 + e)
    assert np.abs(2 * s * _series("kAtanhSeries", s * s) / np.log1p(e) - 1).max() <= 1e-10
