"""rotary_embed up to its largest number of heads, whose count plus a thread's
step between heads passes 2^31."""
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 4097


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def test_the_largest_number_of_heads():
    """One entry a head, which is only converted: FP8 codes stay what they are."""
    say("rotary,", MOST, "heads")
    x = torch.empty((1, MOST, 1), dtype=torch.uint8, device=DEV)
    x.random_(0, 0x7C)
    y = torch.full_like(x, 0xFF)
    none = torch.zeros(0, dtype=torch.float64, device=DEV)
    at = torch.zeros(1, dtype=torch.int64, device=DEV)
    fp8t.rotary_embed(x, at, none, y)
    assert torch.equal(x, y)


def test_turned_heads():
    """Pairs: at position 0 every head is as it was, at position 1 with a
    quarter turn the halves are swapped, one of them negated."""
    H = 2 ** 30 + 12345
    say("rotary,", H, "heads of one pair")
    x = torch.empty((1, H, 2), dtype=torch.uint8, device=DEV)
    x.random_(1, 0x7C)
    y = torch.empty_like(x)
    freqs = torch.tensor([torch.pi / 2], dtype=torch.float64, device=DEV)
    fp8t.rotary_embed(x, torch.zeros(1, dtype=torch.int64, device=DEV), freqs, y)
    assert torch.equal(x, y)
    x[:, :, 1] = x[:, :, 0]                            # (a, a) turns into (-a, a)
    fp8t.rotary_embed(x, torch.ones(1, dtype=torch.int64, device=DEV), freqs, y)
    assert torch.equal(y[:, :, 1], x[:, :, 0]) and torch.equal(y[:, :, 0], x[:, :, 0] | 0x80)
