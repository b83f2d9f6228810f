"""The operators on tokens and rows, called as the documentation allows and the
other tests do not: rows beyond 2^32 bytes, other streams, two calls at once,
captured graphs that share a workspace."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import DEV, dev, host, say
from tests.token_util import F8, F16, F32, TORCH, draw, gpu, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
FAR = 2 ** 31 + 24                       # elements from one row to the next


def far(rows, ty):
    """A matrix whose rows are FAR elements apart, in a buffer that holds them."""
    n, W = len(rows), rows.shape[1]
    buf = torch.empty((n - 1) * FAR + W, dtype=TORCH[ty], device=DEV)
    view = buf.as_strided((n, W), (FAR, 1))
    for i in range(n):                   # row by row: no index kernel over the whole buffer
        view[i].view(torch.int16 if ty == F16 else view.dtype).copy_(
            dev(rows[i]).view(torch.int16) if ty == F16 else dev(rows[i]))
    return view


def rows_of(view):
    return np.stack([host(view[i]) for i in range(len(view))])


def test_rows_far_apart():
    """Strides whose products pass 32 bits: the results of rows beside each other."""
    rng = np.random.default_rng(110)
    say("rows far apart: embedding")
    tok, table = dev(np.array([2, 0, 1, 2])), draw(rng, (3, 40), F8)
    y, want = far(np.zeros((4, 40), F8), F8), torch.empty((4, 40), dtype=torch.uint8, device=DEV)
    fp8t.embed_fwd(tok, dev(table), want, 1.5)
    fp8t.embed_fwd(tok, far(table, F8), y, 1.5)
    assert np.array_equal(rows_of(y), host(want))
    g, want = far(np.zeros((3, 40), F8), F8), torch.empty((3, 40), dtype=torch.uint8, device=DEV)
    e = draw(rng, (4, 40), F8)
    n = fp8t.embed_bwd_workspace_size(tok, dev(e), want)
    fp8t.embed_bwd(tok, dev(e), want, 1.0, workspace(n), n)
    fp8t.embed_bwd(tok, far(e, F8), g, 1.0, workspace(n), n)
    assert np.array_equal(rows_of(g), host(want))
    del y, g
    say("rows far apart: norm")
    x, w = draw(rng, (2, 300), F16), dev(draw(rng, 300, F16))
    h, y = torch.empty((2, 300), dtype=torch.uint16, device=DEV), torch.empty((2, 300), dtype=torch.uint8, device=DEV)
    rstd = torch.empty(2, device=DEV)
    fp8t.rms_norm_fwd(dev(x), dev(x), w, 1e-5, h, y, rstd=rstd)
    fx, fy = far(x, F16), far(np.zeros((2, 300), F8), F8)
    fp8t.rms_norm_fwd(fx, fx, w, 1e-5, fx, fy)
    assert np.array_equal(rows_of(fx), host(h)) and np.array_equal(rows_of(fy), host(y))
    dx, dw = torch.empty_like(h), [torch.empty(300, device=DEV) for _ in range(2)]
    n = fp8t.rms_norm_bwd_workspace_size(h)
    fp8t.rms_norm_bwd(h, w, rstd, y, h, dx, None, 1.0, dw[0], workspace(n), n)
    fd = far(np.zeros((2, 300), F16), F16)
    fp8t.rms_norm_bwd(fx, w, rstd, fy, fx, fd, None, 1.0, dw[1], workspace(n), n)
    assert np.array_equal(rows_of(fd), host(dx)) and np.array_equal(host(dw[0]), host(dw[1]))
    del fx, fy, fd
    say("rows far apart: log probabilities")
    z, idx = draw(rng, (2, 9000), F16), dev(rng.integers(0, 9000, (2, 2)))
    out = [[torch.empty((2, 2), device=DEV), torch.empty(2, device=DEV), torch.empty((2, 2), device=DEV)]
           for _ in range(2)]
    fz = far(z, F16)
    fp8t.token_logprobs(dev(z), idx, 1.0, *out[0])
    fp8t.token_logprobs(fz, idx, 1.0, *out[1])
    for a, b in zip(*out):
        assert np.array_equal(host(a), host(b))
    g = torch.empty((2, 9000), dtype=torch.uint16, device=DEV)
    fp8t.token_logprobs_bwd(dev(z), idx, 1.0, out[0][2], None, out[0][0], None, 1.0, g)
    fp8t.token_logprobs_bwd(fz, idx, 1.0, out[0][2], None, out[0][0], None, 1.0, fz)
    assert np.array_equal(rows_of(fz), host(g))


def test_results_past_the_caches():
    """Results beyond 32 MB are stored past the caches: rows at odd addresses and
    the tails of rows, against the same rows in a small call."""
    rng = np.random.default_rng(111)
    V, W, T = 50, 1003, 40000
    for ty in (F8, F16, F32):
        say("results past the caches", ty.__name__)
        table, tok = dev(draw(rng, (V, W), F16)), dev(np.tile(rng.integers(-1, V, 400), T // 400))
        y, small = torch.empty((T, W), dtype=TORCH[ty], device=DEV), torch.empty((400, W), dtype=TORCH[ty], device=DEV)
        fp8t.embed_fwd(tok, table, y, 2.0)
        fp8t.embed_fwd(tok[:400].clone(), table, small, 2.0)
        raw = torch.int16 if ty == F16 else y.dtype
        assert bool((y.view(raw).view(T // 400, 400, W) == small.view(raw)).all())
        x = y if ty != F8 else torch.empty((T, W), device=DEV).uniform_(-3, 3)
        if ty == F8:
            x.copy_(x[:400].repeat(T // 400, 1))
        h, n8 = torch.empty_like(x), torch.empty((T, W), dtype=torch.uint8, device=DEV)
        sh, s8 = torch.empty_like(x[:400]), torch.empty((400, W), dtype=torch.uint8, device=DEV)
        fp8t.rms_norm_fwd(x, x, None, 1e-5, h, n8)
        fp8t.rms_norm_fwd(x[:400], x[:400], None, 1e-5, sh, s8)
        raw = torch.int16 if x.dtype == torch.uint16 else x.dtype
        assert bool((h.view(raw).view(T // 400, 400, W) == sh.view(raw)).all())
        assert bool((n8.view(T // 400, 400, W) == s8).all())


def test_streams_and_two_calls_at_once():
    """Calls on another stream than the current one, and overlapping ones with
    workspaces of their own: the results of calls one after the other."""
    rng = np.random.default_rng(112)
    tok, e = dev(rng.integers(0, 3000, 9000)), dev(draw(rng, (9000, 256), F16))
    z, idx = dev(draw(rng, (3, 90000), F16)), dev(rng.integers(0, 90000, (3, 1)))
    h, w = dev(draw(rng, (3000, 700), F32)), dev(draw(rng, 700, F16))
    rstd = torch.ones(3000, device=DEV)
    empty = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device=DEV)

    def calls(stream):
        """Each with its own results and workspaces."""
        g, dx, dw = empty(3000, 256), empty(3000, 700), empty(700)
        top, logp = empty(3, 20, dtype=torch.int64), empty(3, 20)
        ws = [workspace(n) for n in (fp8t.embed_bwd_workspace_size(tok, e, g), fp8t.rms_norm_bwd_workspace_size(h),
                                     fp8t.token_logprobs_workspace_size(z, 20))]
        torch.cuda.synchronize()

        def go():
            fp8t.embed_bwd(tok, e, g, 1.0, ws[0], ws[0].numel(), stream=stream)
            fp8t.rms_norm_bwd(h, w, rstd, h, None, dx, None, 1.0, dw, ws[1], ws[1].numel(), stream=stream)
            fp8t.token_logprobs(z, idx, 1.0, top_idx=top, top_logp=logp, workspace=ws[2],
                                workspace_bytes=ws[2].numel(), stream=stream)
        return go, (g, dx, dw, top, logp)
    go, want = calls(None)
    go()
    want = [host(x).copy() for x in want]
    both = [calls(torch.cuda.Stream()) for _ in range(3)]
    for _ in range(3):
        for go, _ in both:
            go()
    torch.cuda.synchronize()
    for _, got in both:
        for a, b in zip(got, want):
            assert np.array_equal(host(a), b)


def test_graphs_that_share_a_workspace():
    """Two graphs captured with one workspace, replayed in turn on one stream."""
    rng = np.random.default_rng(113)
    sizes, graphs, ws_bytes = ((500, 40), (3000, 900)), [], 0
    made = []
    for T, V in sizes:
        tok, e = dev(rng.integers(0, V, T)), dev(draw(rng, (T, 64), F16))
        g = torch.empty((V, 64), device=DEV)
        ws_bytes = max(ws_bytes, fp8t.embed_bwd_workspace_size(tok, e, g))
        made.append((tok, e, g))
    ws = workspace(ws_bytes)
    want = []
    for tok, e, g in made:
        fp8t.embed_bwd(tok, e, g, 1.0, ws, ws_bytes)
        want.append(host(g).copy())
    side = torch.cuda.Stream()
    for tok, e, g in made:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                fp8t.embed_bwd(tok, e, g, 1.0, ws, ws_bytes)
        graphs.append(graph)
    for i in (0, 1, 1, 0, 1, 0):
        made[i][2].fill_(7.0)
        ws.fill_(0xFF)
        graphs[i].replay()
        assert np.array_equal(host(made[i][2]), want[i])


def test_inputs_change_between_replays():
    """A captured call works on what its inputs hold when it is replayed."""
    rng = np.random.default_rng(114)
    tok, e, g = dev(rng.integers(0, 90, 700)), dev(draw(rng, (700, 64), F16)), torch.empty((90, 64), device=DEV)
    n = fp8t.embed_bwd_workspace_size(tok, e, g)
    ws, side, graph = workspace(n), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    fp8t.embed_bwd(tok, e, g, 1.0, ws, n)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            fp8t.embed_bwd(tok, e, g, 1.0, ws, n)
    for k in (1, 3, 90):
        tok.copy_(dev(rng.integers(0, k, 700)))
        graph.replay()
        got = host(g).copy()
        fp8t.embed_bwd(tok, e, g, 1.0, ws, n)
        assert np.array_equal(got, host(g))
