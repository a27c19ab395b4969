"""Calls at the limits of what include/br_kv.h allows, on the GPU: windows, strides, scales, lists that name a block twice, streams."""
import ctypes as C
import math
import weakref

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests import kv_oracle as ko
from tests.test_kv_gpu import _attend_case, _dev, _say, _scattered, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30, 2 ** 20 + 1, 2 ** 20, 129, 128])
@pytest.mark.parametrize("group", [1, 4])
def test_windows_that_hide_nothing(window, group):
    """Up to the largest number that fits, with rows of fewer tokens than queries: whoever is there sees all tokens up to itself."""
    lens, counts = [[20, 3, 40, 0, 100]], [[30, 9, 2, 3, 4]]  # (tables of 8 blocks of 16 tokens)
    _attend_case("window", "int8", "float16", 64, 2, group, 16, lens, counts, window=window)
    _attend_case("window", "fp8", "bfloat16", 128, 1, group, 16, lens, counts, window=window)
