"""Helpers of the GPU tests of the operators on tokens and rows."""
import numpy as np
import pytest
import torch

import oracle
import paper_1812_08011_amd as fp8t
from tests.gpu_util import DEV, dev, host
from tests.lm_util import codes8, codes16

TORCH = {np.float32: torch.float32, np.uint16: torch.uint16, np.uint8: torch.uint8}
F32, F16, F8 = np.float32, np.uint16, np.uint8
EPS32 = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def draw(rng, shape, ty, std=1.0):
    return (rng.standard_normal(shape) * std).astype(F32) if ty == F32 else \
        codes16(rng, shape, std) if ty == F16 else codes8(rng, shape, std)


def rounded(x, ty, scale=1.0):
    """Codes of float32 values as the library's quantizers round them."""
    x = np.asarray(x, F32) * F32(scale)
    return x if ty == F32 else oracle.fp16_quantize(x) if ty == F16 else oracle.fp8_quantize(x)


class Wide:
    """A rows x cols array inside a wider buffer, whose rest must stay as it is.
    pad, shift: columns behind and before."""

    def __init__(self, rows, cols, ty, pad=0, shift=0, data=None):
        self.at, self.pattern = (slice(None), slice(shift, shift + cols)), 0x5A
        fill = np.full((rows, cols + pad + shift), self.pattern, ty)
        if data is not None:
            fill[self.at] = data
        self.buf = dev(fill)
        self.view = self.buf[:, shift:shift + cols]

    def result(self):
        got = host(self.buf).copy()
        out = got[self.at].copy()
        got[self.at] = self.pattern
        assert (got == self.pattern).all(), "written outside the rows"
        return out


def workspace(n):
    """n bytes, all NaN to start with."""
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if n else None


def replayed(call, results, times=3):
    """The results (host copies) of a call captured into a graph and replayed,
    with eager work in between; each replay against the eager call."""
    call()
    want = [host(r).copy() for r in results]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            call()
    for _ in range(times):
        for r in results:
            (r.view(torch.int16) if r.dtype == torch.uint16 else r).fill_(7)
        graph.replay()
        for r, w in zip(results, want):
            assert np.array_equal(host(r), w, equal_nan=r.dtype == torch.float32)
        call()
        for r, w in zip(results, want):
            assert np.array_equal(host(r), w, equal_nan=r.dtype == torch.float32)
