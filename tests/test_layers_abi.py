"""The layers' entry points without a GPU: sizes of workspaces, and everything that is refused before a launch."""
import ctypes

import pytest
import torch

from paper_2412_18052_b200 import binding
from paper_2412_18052_b200.build import build

# Fake, never dereferenced addresses: the checks below must return before any CUDA call.
A = 0x7000_0000_0000
G = 1 << 32
OK, ARG, ALIGN, ALIAS, WORKSPACE, TOO_LARGE = 0, 1, 2, 3, 4, 8
F32, BF16, I32, I64 = 0, 1, 0, 1


@pytest.fixture(scope="module")
def L():
    build()
    return binding.lib()


def test_workspace_bytes(L):
    out = ctypes.c_size_t()

    def size(T, width, V, dtype):
        assert L.gaf_layer_workspace_bytes(T, width, V, dtype, ctypes.byref(out)) == OK
        assert out.value % 256 == 0
        return out.value
    assert size(0, 0, 0, F32) > 0
    for smaller, larger in (((10, 64, 0), (1000, 64, 0)), ((1000, 64, 0), (1000, 4096, 0)), ((1000, 64, 0), (1000, 64, 10 ** 6))):
        for t in (F32, BF16):
            assert size(*smaller, t) < size(*larger, t)
    assert size(1000, 1000, 0, BF16) < size(1000, 1000, 0, F32)
    for bad in ((-1, 1, 1, F32), (1, -1, 1, F32), (1, 1, -1, F32), (1 << 31, 1, 1, F32), (1, 1 << 31, 1, F32), (1, 1, 1 << 31, F32), (1, 1, 1, 2)):
        assert L.gaf_layer_workspace_bytes(*bad, ctypes.byref(out)) == ARG
    assert L.gaf_layer_workspace_bytes(1, 1, 1, F32, None) == ARG


def test_embedding_refusals(L):
    def call(table=A, stride=64, V=100, d=64, dtype=F32, tokens=A + G, tt=I64, T=10, out=A + 2 * G):
        return L.gaf_embedding(table, stride, V, d, dtype, tokens, tt, T, 1.0, out, None)
    assert call(T=0) == OK and call(d=0, stride=0) == OK          # nothing to do: nothing is launched
    assert call(table=None) == ARG and call(tokens=None) == ARG and call(out=None) == ARG
    assert call(stride=63) == ARG and call(dtype=2) == ARG and call(tt=2) == ARG
    assert call(T=-1) == ARG and call(V=-1) == ARG and call(d=-1) == ARG and call(V=1 << 31) == ARG
    assert call(table=A + 8) == ALIGN and call(out=A + 2 * G + 4) == ALIGN and call(tokens=A + G + 4) == ALIGN
    assert call(tokens=A + G + 2, tt=I32) == ALIGN
    assert call(out=A + 64) == ALIAS and call(out=A + G - 64) == ALIAS


def test_embedding_grad_refusals(L):
    def call(dy=A, stride=64, T=10, d=64, dtype=F32, tokens=A + G, tt=I64, base=None, grad=A + 2 * G, gt=F32, V=100, ws=A + 3 * G, n=1 << 30):
        return L.gaf_embedding_grad(dy, stride, T, d, dtype, tokens, tt, 1.0, base, grad, gt, V, ws, n, None)
    assert call(V=0) == OK and call(d=0, stride=0) == OK
    assert call(dy=None) == ARG and call(tokens=None) == ARG and call(grad=None) == ARG and call(stride=60) == ARG
    assert call(dtype=5) == ARG and call(gt=5) == ARG and call(tt=-1) == ARG and call(T=-1) == ARG
    assert call(dy=A + 4) == ALIGN and call(grad=A + 2 * G + 8) == ALIGN and call(base=A + 4 * G + 8) == ALIGN
    assert call(grad=A + 16) == ALIAS and call(base=A + 2 * G + 16) == ALIAS and call(grad=A + G) == ALIAS
    assert call(ws=None) == WORKSPACE and call(ws=A + 3 * G + 16) == WORKSPACE and call(n=1000) == WORKSPACE


def test_checkpoint_refusals(L):
    def pack(x=A, xs=200, T=10, d=200, dtype=F32, codes=A + G, cs=208, scales=A + 2 * G):
        return L.gaf_checkpoint_pack(x, xs, T, d, dtype, codes, cs, scales, None)

    def unpack(codes=A + G, cs=208, scales=A + 2 * G, T=10, d=200, dtype=F32, out=A, os=200):
        return L.gaf_checkpoint_unpack(codes, cs, scales, T, d, dtype, out, os, None)
    for f in (pack, unpack):
        assert f(T=0) == OK
        assert f(codes=None) == ARG and f(scales=None) == ARG and f(cs=192) == ARG and f(dtype=3) == ARG and f(T=-2) == ARG
        assert f(cs=201) == ALIGN and f(codes=A + G + 8) == ALIGN and f(scales=A + 2 * G + 1) == ALIGN
        assert f(codes=A + 160) == ALIAS
    assert pack(x=None) == ARG and pack(xs=199) == ARG and pack(x=A + 2) == ALIGN and pack(scales=A + G + 16) == ALIAS
    assert unpack(out=None) == ARG and unpack(os=199) == ARG and unpack(out=A + 2) == ALIGN


def test_rms_norm_refusals(L):
    def call(x=A, xs=64, res=None, rs=64, w=A + G, T=10, d=64, dtype=F32, eps=1e-6, h=None, y=A + 2 * G, yc=None, ycs=64, ysc=None, coded=0,
             hc=None, hcs=64, hsc=None, rstd=A + 3 * G):
        return L.gaf_rms_norm(x, xs, res, rs, w, T, d, dtype, eps, h, y, yc, ycs, ysc, coded, hc, hcs, hsc, rstd, None)
    assert call(T=0) == OK
    assert call(x=None) == ARG and call(w=None) == ARG and call(xs=10) == ARG and call(d=0) == ARG and call(T=-1) == ARG and call(dtype=2) == ARG
    assert call(eps=-1.0) == ARG and call(eps=float("nan")) == ARG and call(eps=float("inf")) == ARG
    assert call(h=A + 4 * G) == ARG                                # h without a residual is x
    assert call(yc=A + 5 * G) == ARG and call(ysc=A + 5 * G) == ARG and call(hc=A + 5 * G) == ARG and call(coded=1) == ARG
    assert call(y=None, rstd=None) == ARG                          # no output at all
    assert call(y=None, coded=1, yc=A + 5 * G, ysc=A + 6 * G) == ARG
    assert call(d=16385, xs=16385) == TOO_LARGE
    assert call(yc=A + 5 * G, ysc=A + 6 * G, ycs=72) == ALIGN and call(x=A + 4) == ALIGN and call(y=A + 2 * G + 4) == ALIGN and call(rstd=A + 3 * G + 4) == ALIGN
    assert call(y=A) == ALIAS and call(res=A + 4 * G, h=A + 4 * G + 64) == ALIAS and call(res=A + 4 * G, rs=72, h=A + 4 * G) == ALIAS
    assert call(y=A + G) == ALIAS and call(rstd=A + 2 * G) == ALIAS and call(res=A + 4 * G, h=A + 2 * G) == ALIAS


def test_rms_norm_grad_refusals(L):
    def call(dy=A, ds=64, h=A + G, hs=64, hc=None, hcs=64, hsc=None, w=A + 2 * G, rstd=A + 3 * G, res=None, rs=64, T=10, d=64, dtype=F32, dx=A + 4 * G,
             base=None, dw=A + 5 * G, gt=F32, ws=A + 6 * G, n=1 << 30):
        return L.gaf_rms_norm_grad(dy, ds, h, hs, hc, hcs, hsc, w, rstd, res, rs, T, d, dtype, dx, base, dw, gt, ws, n, None)
    assert call(dy=None) == ARG and call(h=None) == ARG and call(hc=A + 7 * G, hsc=A + 8 * G) == ARG and call(w=None) == ARG and call(rstd=None) == ARG
    assert call(dx=None) == ARG and call(dw=None) == ARG and call(gt=4) == ARG and call(dtype=4) == ARG and call(d=0) == ARG
    assert call(h=None, hc=A + 7 * G) == ARG and call(ds=32) == ARG and call(res=A + 9 * G, rs=8) == ARG
    assert call(d=20000, ds=20000, hs=20000) == TOO_LARGE
    assert call(dy=A + 4) == ALIGN and call(dw=A + 5 * G + 4) == ALIGN and call(h=None, hc=A + 7 * G, hsc=A + 8 * G, hcs=65) == ALIGN
    assert call(dx=A + G) == ALIAS and call(dx=A + 16) == ALIAS and call(dw=A + 4 * G) == ALIAS and call(dw=A + 2 * G) == ALIAS
    assert call(ws=None) == WORKSPACE and call(n=4096) == WORKSPACE


def test_linear_weight_grad_refusals(L):
    def call(dy=A, ds=64, dtype=BF16, codes=A + G, cs=128, scales=A + 2 * G, T=10, N=64, M=128, base=None, dw=A + 3 * G, gt=F32, ws=A + 4 * G, n=1 << 30):
        return L.gaf_linear_weight_grad(dy, ds, dtype, codes, cs, scales, T, N, M, base, dw, gt, ws, n, None)
    assert call(N=0) == OK and call(M=0) == OK
    assert call(dy=None) == ARG and call(codes=None) == ARG and call(scales=None) == ARG and call(dw=None) == ARG
    assert call(ds=63) == ARG and call(cs=112) == ARG and call(dtype=2) == ARG and call(gt=2) == ARG and call(T=-1) == ARG and call(N=-1) == ARG
    assert call(cs=136) == ALIGN and call(dy=A + 8) == ALIGN and call(base=A + 5 * G + 4) == ALIGN
    assert call(dw=A) == ALIAS and call(dw=A + G + 16) == ALIAS and call(base=A + 3 * G + 16) == ALIAS


def test_binding_refuses_host_tensors():
    """Tensors that are not on the current CUDA device are refused, not read."""
    x, w, ws = torch.zeros(4, 64), torch.zeros(64), torch.zeros(1 << 12, dtype=torch.uint8)
    tokens, ck = torch.zeros(4, dtype=torch.int64), (torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8))
    calls = [lambda: binding.gaf_embedding(x, tokens), lambda: binding.gaf_embedding_grad(x, tokens, x, ws),
             lambda: binding.gaf_checkpoint_pack(x, ck), lambda: binding.gaf_checkpoint_unpack(ck, out=x),
             lambda: binding.gaf_rms_norm(x, w), lambda: binding.gaf_rms_norm_grad(x, x, w, torch.zeros(4), w, ws),
             lambda: binding.gaf_linear_weight_grad(x, ck, torch.zeros(64, 64), ws)]
    for call in calls:
        with pytest.raises(ValueError, match="CUDA device"):
            call()
    with pytest.raises(TypeError):
        binding.gaf_embedding("x", tokens)
