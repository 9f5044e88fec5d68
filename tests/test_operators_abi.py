"""Refusals of the operators' C entry points, on the host before any CUDA call."""
import ctypes

import pytest

import paper_2608_06291_gb300 as P

FAKE = ctypes.c_void_p(0x1000)   # never dereferenced: validation fails first
F32, BF16, E4M3 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    P.build()
    return P.lib()


def _with(base, **changed):
    args = dict(base)
    args.update(changed)
    return list(args.values())


def test_pack_weight(L):
    ok = dict(codes=FAKE, ldc=64, scales=FAKE, zeros=FAKE, m=8, n=64, qmax=15, group=32, packed=FAKE, bytes=1 << 30,
              stream=None)
    for bad in (dict(codes=None), dict(scales=None), dict(zeros=None), dict(packed=None), dict(ldc=63), dict(m=0),
                dict(n=0), dict(qmax=0), dict(qmax=256), dict(group=16), dict(group=48), dict(group=-32),
                dict(m=(1 << 17) + 1), dict(packed=ctypes.c_void_p(0x1001))):
        assert L.bakron_pack_weight(*_with(ok, **bad)) == 1, bad
    assert L.bakron_pack_weight(*_with(ok, bytes=255)) == 5
    assert L.bakron_packed_bytes(8, 64, 15, 24) == 0
    # 4 bits a code in whole blocks of 128 x 128, 8 above qmax 15
    four, eight = L.bakron_packed_bytes(1000, 1000, 15, 0), L.bakron_packed_bytes(1000, 1000, 16, 0)
    assert 1024 * 512 <= four < 1024 * 512 + 8192 and eight - four == 1024 * 512


def test_linear(L):
    ok = dict(x=FAKE, xdtype=BF16, rows=4, ldx=64, xscales=None, packed=FAKE, m=8, n=64, qmax=15, group=32, bias=None,
              activation=0, residual=None, ldr=0, y=FAKE, ydtype=BF16, ldy=8, ws=None, ws_bytes=0, sync=0, stream=None)
    for bad in (dict(x=None), dict(xdtype=F32), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(ldx=63), dict(packed=None), dict(m=0), dict(n=0),
                dict(qmax=0), dict(group=16), dict(activation=4), dict(activation=-1), dict(residual=FAKE, ldr=7),
                dict(y=None), dict(ydtype=E4M3), dict(ldy=7), dict(packed=ctypes.c_void_p(0x1008))):
        assert L.bakron_linear(*_with(ok, **bad)) == 1, bad
    assert L.bakron_linear(*_with(ok, rows=0, x=None, y=None, packed=None)) == 0


def test_rmsnorm(L):
    ok = dict(x=FAKE, dtype=BF16, rows=4, d=64, ldx=64, residual=None, ldr=0, weight=FAKE, wdtype=F32,
              eps=ctypes.c_float(1e-5), sum=None, lds=0, y=FAKE, ydtype=BF16, ldy=64, scales=None, stream=None)
    for bad in (dict(x=None), dict(dtype=E4M3), dict(rows=-1), dict(d=0), dict(d=65537), dict(ldx=63),
                dict(residual=FAKE, ldr=63), dict(weight=None), dict(wdtype=E4M3), dict(eps=ctypes.c_float(-1.0)),
                dict(eps=ctypes.c_float(float("nan"))), dict(sum=FAKE, lds=63), dict(y=None), dict(ydtype=F32),
                dict(ydtype=E4M3), dict(ldy=63)):
        assert L.bakron_rmsnorm(*_with(ok, **bad)) == 1, bad
    assert L.bakron_rmsnorm(*_with(ok, rows=0, x=None)) == 0
    back = dict(dy=FAKE, lddy=64, h=FAKE, ldh=64, dtype=F32, rows=4, d=64, weight=FAKE, wdtype=F32,
                eps=ctypes.c_float(1e-5), dsum=None, ldds=0, dx=FAKE, lddx=64, dw=FAKE, ws=FAKE, bytes=1 << 30,
                stream=None)
    for bad in (dict(dy=None), dict(h=None), dict(lddy=63), dict(ldh=63), dict(dtype=E4M3), dict(rows=-1), dict(d=0),
                dict(weight=None), dict(wdtype=3), dict(dsum=FAKE, ldds=63), dict(dx=None), dict(lddx=63),
                dict(dw=None), dict(ws=None), dict(eps=ctypes.c_float(-1.0))):
        assert L.bakron_rmsnorm_backward(*_with(back, **bad)) == 1, bad
    assert L.bakron_rmsnorm_backward(*_with(back, bytes=16)) == 5


def test_token_logprobs(L):
    ok = dict(logits=FAKE, dtype=BF16, rows=4, v=100, ldl=100, targets=FAKE, top=5, logp=FAKE, entropy=FAKE, lse=FAKE,
              top_logp=FAKE, top_ids=FAKE, stream=None)
    for bad in (dict(logits=None), dict(dtype=E4M3), dict(rows=-1), dict(v=0), dict(ldl=99), dict(top=-1), dict(top=33),
                dict(top=5, v=4), dict(targets=None), dict(logp=None), dict(entropy=None), dict(lse=None),
                dict(top_logp=None), dict(top_ids=None)):
        assert L.bakron_token_logprobs(*_with(ok, **bad)) == 1, bad
    assert L.bakron_token_logprobs(*_with(ok, rows=0, logits=None)) == 0
    back = dict(logits=FAKE, dtype=F32, rows=4, v=100, ldl=100, targets=FAKE, lse=FAKE, dlogp=FAKE, entropy=None,
                dentropy=None, dlogits=FAKE, ldd=100, stream=None)
    for bad in (dict(logits=None), dict(dtype=E4M3), dict(rows=-1), dict(v=0), dict(ldl=99), dict(ldd=99),
                dict(targets=None), dict(lse=None), dict(dlogp=None), dict(dentropy=FAKE), dict(dlogits=None)):
        assert L.bakron_token_logprobs_backward(*_with(back, **bad)) == 1, bad
