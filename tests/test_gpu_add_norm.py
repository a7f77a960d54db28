"""Residual addition + norm + INT8 quantizer in one pass against a plain evaluation: binary64 statistics,
binary32 elements, bit for bit."""

import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from util import Guarded

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def plain(X, res, w, b, layer, eps):
    """numpy, one rounding per operation."""
    f = np.float32
    y = torch.from_numpy(X.float().numpy() + res.float().numpy()).to(res.dtype)
    x = y.float().numpy()
    K = x.shape[1]
    if layer:
        x = x - (x.astype(np.float64).sum(1, keepdims=True) / K).astype(f)
    x64 = x.astype(np.float64)
    r = (1.0 / np.sqrt((x64 * x64).sum(1, keepdims=True) / K + float(f(eps)))).astype(f)
    x = (x * r) * w
    if b is not None:
        x = x + b
    amax = np.abs(x).max(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.rint(np.clip(x * (f(127) / amax), f(-127), f(127)))
    q = np.where(amax > 0, q, 0).astype(np.int8)
    return q, (amax / f(127))[:, 0], y


def run(M, K, kind, bias, x_type, res_type, seed, in_place=False, mutate=None, eps=1e-5):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(M, K, generator=g).to(TYPES[x_type])
    res = (torch.randn(M, K, generator=g) * (1 + 19 * (torch.rand(K, generator=g) < 0.02)) + 0.3).to(TYPES[res_type])
    if mutate is not None:
        mutate(X, res)
    w = torch.exp(0.7 * torch.randn(K, generator=g))
    b = 0.1 * torch.randn(K, generator=g) if bias else None
    q, t, y = plain(X, res, w.numpy(), None if b is None else b.numpy(), kind == "layer", eps)
    gq, gt, gr = Guarded((M, K), torch.int8), Guarded((M,), torch.float32), Guarded((M, K), TYPES[res_type])
    gr.t.copy_(res)
    src = gr.t if in_place else res.cuda()
    code = w4a8.NORM_LAYER if kind == "layer" else w4a8.NORM_RMS
    w4a8.add_norm_quantize_act(X.cuda(), src, w.cuda(), None if b is None else b.cuda(), code, eps,
                               residual_out=gr.t, out=(gq.t, gt.t))
    for buf, what in ((gq, "Xq"), (gt, "tok_scale"), (gr, "residual_out")):
        buf.check(what)
    assert torch.equal(gr.t.cpu(), y)
    assert np.array_equal(gt.t.cpu().numpy().view(np.uint32), t.view(np.uint32))
    assert np.array_equal(gq.t.cpu().numpy(), q)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M,K", [(1, 128), (16, 768), (37, 1152), (300, 4096), (5, 16384), (1, 9216), (3, 8320)])
def test_sizes(kind, bias, M, K):
    run(M, K, kind, bias, "bf16", "f16", M + K)


@pytest.mark.parametrize("x_type", ["f16", "bf16"])
@pytest.mark.parametrize("res_type", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("in_place", [False, True])
def test_types(x_type, res_type, kind, in_place):
    run(11, 2048, kind, kind == "layer", x_type, res_type, 7, in_place)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_zero_constant_small_and_large_tokens(kind):
    def mutate(X, res):
        X[0], res[0] = 0, 0
        X[1], res[1] = 1.0, 2.0
        X[2], res[2] = -res[2].to(X.dtype), -(-res[2].to(X.dtype)).to(res.dtype)     # cancels to zero
        X[3] *= 1e-4
        res[3] *= 1e-4
        X[4] *= 1e3
        res[4] *= 1e3

    for bias in (False, True):
        run(6, 1024, kind, bias, "f16", "f16", 3, mutate=mutate)
        run(6, 1024, kind, bias, "bf16", "f32", 4, mutate=mutate, eps=1e-6)


def test_magnitudes_beyond_binary32_squares():
    """A 32-bit stream of 1e25: its squares do not fit binary32, its statistics do."""
    def mutate(X, res):
        res *= 1e25
    run(4, 512, "rms", False, "bf16", "f32", 5, mutate=mutate)
    run(4, 512, "layer", True, "bf16", "f32", 6, mutate=mutate)


def test_many_rows():
    run(3001, 512, "rms", False, "bf16", "bf16", 1)


def test_agrees_with_the_unfused_calls_on_the_stored_sum():
    """addition, then w4a8_norm_quantize_act: the root may differ by one binary32 step, a code then by one."""
    X, res = torch.randn(64, 4096).cuda().half(), torch.randn(64, 4096).cuda().half()
    w = torch.rand(4096, device="cuda") + 0.5
    Xq, tok, y = w4a8.add_norm_quantize_act(X, res, w)
    Xq2, tok2 = w4a8.norm_quantize_act(y, w)
    assert bool(((Xq.int() - Xq2.int()).abs() <= 1).all())
    assert bool(((tok - tok2).abs() <= 2.0 ** -22 * tok).all())


def test_graph_replay_and_refusals():
    X, res = torch.randn(8, 256).cuda().half(), torch.randn(8, 256).cuda()
    w = torch.ones(256, device="cuda")
    want = w4a8.add_norm_quantize_act(X, res, w)
    out = (torch.empty_like(want[0]), torch.empty_like(want[1]))
    ro, graph = torch.empty_like(res), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w4a8.add_norm_quantize_act(X, res, w, residual_out=ro, out=out)
    graph.replay()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(ro, want[2])
    with pytest.raises(TypeError):
        w4a8.add_norm_quantize_act(X.float(), res, w)
    with pytest.raises(ValueError):
        w4a8.add_norm_quantize_act(X, res[:4], w)
    with pytest.raises(TypeError):
        w4a8.add_norm_quantize_act(X, res[:, ::2], w)
