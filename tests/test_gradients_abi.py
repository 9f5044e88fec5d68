"""Refusals of the head's, the layer norm's and the product gradient's C entry points, on the host before any
CUDA call; their workspaces."""
import ctypes

import pytest
import torch

import paper_2608_06291_gb300 as P

FAKE = ctypes.c_void_p(0x1000)   # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)
F32, BF16, E4M3 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    P.build()
    return P.lib()


def _with(base, **changed):
    args = dict(base)
    args.update(changed)
    return list(args.values())


def test_head_logprobs(L):
    ok = dict(h=FAKE, ldh=64, weight=FAKE, ldw=64, rows=4, v=100, d=64, targets=FAKE, logp=FAKE, entropy=FAKE, lse=FAKE,
              ws=FAKE, bytes=1 << 30, sync=0, stream=None)
    for bad in (dict(h=None), dict(ldh=63), dict(weight=None), dict(ldw=63), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(v=0),
                dict(v=(1 << 24) + 1), dict(d=0), dict(d=65537), dict(targets=None), dict(logp=None), dict(entropy=None),
                dict(lse=None), dict(ws=None), dict(ws=ctypes.c_void_p(0x1008)), dict(h=ODD), dict(weight=ODD)):
        assert L.bakron_head_logprobs(*_with(ok, **bad)) == 1, bad
    need = L.bakron_head_logprobs_workspace_bytes(FAKE, 64, FAKE, 64, 4, 100, 64)
    assert L.bakron_head_logprobs(*_with(ok, bytes=need - 1)) == 5
    assert L.bakron_head_logprobs(*_with(ok, rows=0, h=None)) == 0
    # what cannot be read in place is copied: 100 rows of 64 values
    assert L.bakron_head_logprobs_workspace_bytes(FAKE, 64, FAKE, 65, 4, 100, 64) == need + 100 * 128
    assert L.bakron_head_logprobs_workspace_bytes(FAKE, 64, FAKE, 64, 4, 0, 64) == 0


def test_head_logprobs_backward(L):
    ok = dict(h=FAKE, ldh=64, weight=FAKE, ldw=64, rows=4, v=100, d=64, targets=FAKE, lse=FAKE, dlogp=FAKE, entropy=None,
              dentropy=None, dh=FAKE, lddh=64, dweight=FAKE, lddw=64, ws=FAKE, bytes=1 << 30, sync=0, stream=None)
    for bad in (dict(h=None), dict(ldh=63), dict(weight=None), dict(ldw=63), dict(rows=-1), dict(v=0), dict(d=0),
                dict(targets=None), dict(lse=None), dict(dentropy=FAKE), dict(dh=None), dict(lddh=63), dict(lddw=63),
                dict(ws=None), dict(ws=ctypes.c_void_p(0x1004)), dict(h=ODD), dict(weight=ODD)):
        assert L.bakron_head_logprobs_backward(*_with(ok, **bad)) == 1, bad
    for given in (0, 1):
        need = L.bakron_head_logprobs_backward_workspace_bytes(FAKE, 64, FAKE, 64, 4, 100, 64, given)
        assert L.bakron_head_logprobs_backward(*_with(ok, dweight=FAKE if given else None, bytes=need - 1)) == 5
    assert L.bakron_head_logprobs_backward(*_with(ok, rows=0, h=None, dweight=None)) == 0


def test_layernorm(L):
    ok = dict(x=FAKE, dtype=BF16, rows=4, d=64, ldx=64, residual=None, ldr=0, weight=FAKE, wdtype=F32, bias=None, bdtype=0,
              eps=ctypes.c_float(1e-5), sum=None, lds=0, y=FAKE, ydtype=BF16, ldy=64, scales=None, stream=None)
    for bad in (dict(x=None), dict(dtype=E4M3), dict(rows=-1), dict(d=0), dict(d=65537), dict(ldx=63),
                dict(residual=FAKE, ldr=63), dict(weight=None), dict(wdtype=E4M3), dict(bias=FAKE, bdtype=E4M3),
                dict(eps=ctypes.c_float(-1.0)), dict(eps=ctypes.c_float(float("nan"))), dict(sum=FAKE, lds=63),
                dict(y=None), dict(ydtype=F32), dict(ydtype=E4M3), dict(ldy=63)):
        assert L.bakron_layernorm(*_with(ok, **bad)) == 1, bad
    assert L.bakron_layernorm(*_with(ok, rows=0, x=None)) == 0
    back = dict(dy=FAKE, lddy=64, h=FAKE, ldh=64, dtype=F32, rows=4, d=64, weight=FAKE, wdtype=F32,
                eps=ctypes.c_float(1e-5), dsum=None, ldds=0, dx=FAKE, lddx=64, dw=FAKE, db=FAKE, ws=FAKE, bytes=1 << 30,
                stream=None)
    for bad in (dict(dy=None), dict(h=None), dict(lddy=63), dict(ldh=63), dict(dtype=E4M3), dict(rows=-1), dict(d=0),
                dict(weight=None), dict(wdtype=3), dict(dsum=FAKE, ldds=63), dict(dx=None), dict(lddx=63),
                dict(dw=None), dict(db=None), dict(ws=None), dict(ws=ctypes.c_void_p(0x1004)), dict(eps=ctypes.c_float(-1.0))):
        assert L.bakron_layernorm_backward(*_with(back, **bad)) == 1, bad
    assert L.bakron_layernorm_backward(*_with(back, bytes=L.bakron_layernorm_backward_workspace_bytes(4, 64) - 1)) == 5


def test_linear_backward(L):
    ok = dict(dy=FAKE, rows=4, lddy=64, packed=FAKE, m=64, n=96, qmax=15, group=32, dx=FAKE, lddx=96, ws=FAKE,
              bytes=1 << 30, sync=0, stream=None)
    for bad in (dict(dy=None), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(lddy=63), dict(packed=None), dict(m=0), dict(n=0),
                dict(m=(1 << 17) + 1), dict(qmax=0), dict(qmax=256), dict(group=16), dict(group=64), dict(dx=None),
                dict(lddx=95), dict(ws=None), dict(ws=ctypes.c_void_p(0x1008)), dict(packed=ctypes.c_void_p(0x1008)),
                dict(dy=ODD), dict(dx=ODD)):
        assert L.bakron_linear_backward(*_with(ok, **bad)) == 1, bad
    for rows in (4, 1000):
        need = L.bakron_linear_backward_workspace_bytes(FAKE, rows, 64, 64, 96, 15, 32)
        assert L.bakron_linear_backward(*_with(ok, rows=rows, bytes=need - 1)) == 5
    assert L.bakron_linear_backward(*_with(ok, rows=0, dy=None)) == 0


def test_the_binding_refuses_on_the_cpu():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64)
    for call in (lambda: P.bakron_head_logprobs(x, x), lambda: P.bakron_head_logprobs_backward(x, x, None, w, None),
                 lambda: P.bakron_layernorm(x, w), lambda: P.bakron_layernorm_backward(x, x, w)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_too_many_rows_are_refused():
    one = torch.ones(1, 1, device="cuda")
    many, few = one.expand(2 ** 32, 1), one.bfloat16()       # without its memory
    w = P.bakron_pack_weight(torch.ones(1, 1, dtype=torch.uint8, device="cuda"), one, one * 0, 1)
    for call in (lambda: P.bakron_linear_backward(few.expand(2 ** 32, 1), w), lambda: P.bakron_layernorm(many, one[0]),
                 lambda: P.bakron_layernorm_backward(many, many, one[0]),
                 lambda: P.bakron_head_logprobs(few.expand(2 ** 32, 1), few)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(P.BakronError):
        P.bakron_head_logprobs(few.expand(2 ** 24 + 1, 1), few)
