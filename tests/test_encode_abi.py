"""Refusals of the prompt encoder's entry points, before any device work (CPU only)."""
import ctypes
import math
import os

import pytest

from paper_2603_07917_amd import sage

SAGE_OK, SAGE_EINVAL, SAGE_EWORKSPACE = 0, -1, -2
P = [0x10000000 * (i + 1) for i in range(12)]            # far apart, aligned, never read


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sage.library_path()):
        from paper_2603_07917_amd import build
        build.build()
    return sage.load_library()


def embed(lib, tokens=P[0], T=100, table=P[1], ttype=1, V=50, d=64, scale=1.0, offsets=P[2], Q=4, mean=0, out=P[3],
          otype=0, ws=P[4], ws_bytes=1 << 30):
    return lib.sage_embed(tokens, T, table, ttype, V, d, scale, offsets, Q, mean, out, otype, ws, ws_bytes, None)


def embed_grad(lib, tokens=P[0], T=100, grad=P[1], gtype=1, V=50, d=64, scale=1.0, offsets=P[2], Q=4, mean=0, add=P[5],
               out=P[3], ws=P[4], ws_bytes=1 << 30):
    return lib.sage_embed_grad(tokens, T, grad, gtype, V, d, scale, offsets, Q, mean, add, out, ws, ws_bytes, None)


def norm(lib, x=P[0], r=P[1], t=1, M=9, d=64, gain=P[2], eps=1e-6, total=P[3], out=P[4], otype=2, scales=P[5]):
    return lib.sage_rms_norm(x, r, t, M, d, gain, eps, total, out, otype, scales, None)


def norm_grad(lib, g=P[0], total=P[1], t=1, M=9, d=64, gain=P[2], eps=1e-6, gt=P[3], gx=P[4], gg=P[5], ws=P[6], ws_bytes=1 << 30):
    return lib.sage_rms_norm_grad(g, total, t, M, d, gain, eps, gt, gx, gg, ws, ws_bytes, None)


def quantize(lib, x=P[0], t=0, M=9, K=64, block=0, transpose=0, q=P[1], scales=P[2]):
    return lib.sage_quantize(x, t, M, K, block, transpose, q, scales, None)


def matmul(lib, a=P[0], sa=P[1], M=9, b=P[2], sb=P[3], block=1, N=33, K=64, bias=P[4], relu=0, out=P[5], otype=1, ws=P[6],
           ws_bytes=1 << 30):
    return lib.sage_matmul_fp8(a, sa, M, b, sb, block, N, K, bias, relu, 0, out, otype, ws, ws_bytes, None)


@pytest.mark.parametrize("call,bad", [
    (embed, [dict(T=-1), dict(T=(1 << 30) + 1), dict(V=0), dict(d=0), dict(d=(1 << 20) + 1), dict(Q=-1), dict(ttype=2),
             dict(otype=2), dict(otype=-1), dict(scale=math.nan), dict(scale=math.inf), dict(offsets=None, mean=1),
             dict(tokens=None), dict(table=None), dict(out=None), dict(tokens=P[0] + 4), dict(table=P[1] + 8),
             dict(offsets=P[2] + 4), dict(out=P[3] + 2), dict(out=P[1] + 16), dict(ws=P[4] + 8)]),
    (embed_grad, [dict(T=-1), dict(V=0), dict(d=0), dict(Q=-1), dict(gtype=2), dict(scale=math.nan), dict(offsets=None, mean=1),
                  dict(tokens=None), dict(grad=None), dict(out=None), dict(add=P[5] + 4), dict(out=P[1]), dict(out=P[5] + 16),
                  dict(out=P[3] + 4)]),
    (norm, [dict(M=-1), dict(d=0), dict(d=32769), dict(t=2), dict(otype=3), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
            dict(x=None), dict(gain=None), dict(out=None), dict(scales=None), dict(x=P[0] + 2), dict(r=P[1] + 8),
            dict(total=P[3] + 4), dict(out=P[0]), dict(out=P[1]), dict(out=P[3]), dict(total=P[0] + 16)]),
    (norm_grad, [dict(M=-1), dict(d=0), dict(t=2), dict(eps=-1.0), dict(g=None), dict(total=None), dict(gain=None), dict(gx=None),
                 dict(gg=None), dict(gt=P[3] + 2), dict(gx=P[0] + 16)]),
    (quantize, [dict(t=2), dict(block=2), dict(M=-1), dict(K=-1), dict(M=1 << 28, K=1), dict(x=None), dict(q=None), dict(scales=None),
                dict(x=P[0] + 4), dict(q=P[0] + 16)]),
    (matmul, [dict(M=-1), dict(N=-1), dict(K=0), dict(K=8), dict(K=100), dict(K=(1 << 20) + 16), dict(block=2), dict(otype=2),
              dict(M=1 << 20, N=1 << 20), dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(out=None), dict(bias=P[4] + 4),
              dict(out=P[5] + 8), dict(out=P[0]), dict(out=P[2])]),
])
def test_refuses(lib, call, bad):
    for kw in bad:
        assert call(lib, **kw) == SAGE_EINVAL, kw
        assert lib.sage_last_error() != b"", kw


def test_small_workspaces(lib):
    need = lib.sage_embed_workspace_bytes(100, 4, 64)
    assert need > 0
    assert embed(lib, ws_bytes=need - 1) == SAGE_EWORKSPACE and embed(lib, ws=None) == SAGE_EWORKSPACE
    need = lib.sage_embed_grad_workspace_bytes(100, 4, 50, 64)
    assert embed_grad(lib, ws_bytes=need - 1) == SAGE_EWORKSPACE and embed_grad(lib, ws=None) == SAGE_EWORKSPACE
    need = lib.sage_rms_norm_grad_workspace_bytes(9, 64)
    assert norm_grad(lib, ws_bytes=need - 1) == SAGE_EWORKSPACE and norm_grad(lib, ws=None) == SAGE_EWORKSPACE
    need = lib.sage_matmul_fp8_workspace_bytes(256, 256, 16384)
    assert need > 0 and matmul(lib, M=256, N=256, K=16384, ws_bytes=need - 1) == SAGE_EWORKSPACE
    for bad in [(-1, 4, 64), (1, -1, 64), (1, 1, 0)]:
        assert lib.sage_embed_workspace_bytes(*bad) == 0
    assert lib.sage_embed_grad_workspace_bytes(1, 1, 0, 8) == 0
    assert lib.sage_rms_norm_grad_workspace_bytes(0, 8) == 0
    assert lib.sage_matmul_fp8_workspace_bytes(0, 8, 16) == 0 and lib.sage_matmul_fp8_workspace_bytes(8, 8, 8) == 0


def test_nothing_to_do(lib):
    assert embed(lib, T=0, offsets=None, tokens=None) == SAGE_OK
    assert embed(lib, Q=0, out=None) == SAGE_OK
    assert norm(lib, M=0, x=None, out=None) == SAGE_OK
    assert quantize(lib, M=0, x=None) == SAGE_OK and quantize(lib, K=0, q=None) == SAGE_OK
    assert matmul(lib, M=0, a=None) == SAGE_OK and matmul(lib, N=0, out=None) == SAGE_OK


def test_python_refuses_host_tensors_and_shapes():
    import torch
    x = torch.zeros(4, 16)
    for call in (lambda: sage.embed(torch.zeros(3, dtype=torch.int32), x), lambda: sage.rms_norm(x, torch.ones(16)),
                 lambda: sage.quantize(x), lambda: sage.quantize(x.half()),
                 lambda: sage.embed_grad(torch.zeros(3, dtype=torch.int32), x, 5),
                 lambda: sage.rms_norm_grad(x, x, torch.ones(16)),
                 lambda: sage.matmul_fp8(x, x, x, x)):
        with pytest.raises(sage.SageError):
            call()


def test_python_refuses_workspaces_elsewhere():
    import torch
    here, meta = torch.device("cpu"), torch.empty(64, dtype=torch.uint8, device="meta")
    ws = torch.empty(64, dtype=torch.uint8)
    assert sage._scratch(ws, 64, here) is ws and sage._scratch(ws, 65, here).numel() == 65
    for bad in (meta, torch.empty(128, dtype=torch.uint8)[::2]):
        for need in (0, 64):
            with pytest.raises(sage.SageError):
                sage._scratch(bad, need, here)
