"""The polynomial behind capped scores of packed chunks (csrc/chunk_device.hpp), without a GPU."""
import os
import re

import numpy as np
import pytest


HERE = os.path.dirname(os.path.abspath(__file__))
SOURCE = open(os.path.join(HERE, "..", "paper_2507_03153_amd", "csrc", "chunk_device.hpp")).read()


@pytest.mark.parametrize("name,degree", [("kFine", 5), ("kCoarse", 4)])
def test_fit_of_the_tanh(name, degree):
    """The coefficients, as fp32 has them, in 64 bits: the largest relative error up to 0.7 is the one that the comment beside them names; the fine
    ones are exact at 0."""
    k = [np.float64(np.float32(x)) for x in re.search(name + r"\[6\] = \{([^}]*)\}", SOURCE).group(1).replace("f", "").split(",")]
    x = np.concatenate([np.linspace(1e-4, 0.7, 200001), [1e-12, 1e-8]])
    err = np.abs(x * sum(c * x ** (2 * i) for i, c in enumerate(k)) / np.tanh(x) - 1).max()
    named = float(re.search(r"([\d.]+e-\d+) of degree %d" % degree, SOURCE).group(1))
    print(name, err, named)
    assert 0.9 * named <= err <= 1.01 * named
    assert name != "kFine" or k[0] == 1
