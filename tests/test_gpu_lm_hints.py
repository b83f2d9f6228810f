"""Attention with size hints far above the call's sizes: results are those of
the definition under the plans that such hints choose."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.test_gpu_attention import both

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


@pytest.mark.parametrize("max_k", [2 ** 31 - 1, 2 ** 38, 2 ** 40, 2 ** 63 - 1])
@pytest.mark.parametrize("max_q", [1, 300, 2 ** 62, 2 ** 63 - 1])
@pytest.mark.parametrize("D", [64, 128])
def test_huge_hints(D, max_q, max_k):
    both(2600 + D, [40, 1], [300, 70], 2, 1, D, True, max_q=max_q, max_k=max_k)
