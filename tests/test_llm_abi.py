"""The entry points of include/attnfuse_llm.h reject bad arguments before any HIP call (CPU tests; no compute calls)."""
import ctypes
import os
import re

import pytest

from paper_2609_13612_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x100000     # aligned, never dereferenced: validation fails first
ODD = 0x100008
TABLE = 0x400000
INVALID, UNSUPPORTED = -1, -2
NAN, INF = float("nan"), float("inf")


def test_header_and_signatures_agree():
    with open(os.path.join(ROOT, "include", "attnfuse_llm.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = dict(re.findall(r"\b(attnfuse_\w+)\s*\(([^)]*)\)", text))
    assert set(declared) == set(_lib.LLM_SIGNATURES)
    lib = _lib.load()
    kinds = {"int": ctypes.c_int, "float": ctypes.c_float, "long long": ctypes.c_longlong, "size_t": ctypes.c_size_t}
    for name, args in declared.items():
        assert hasattr(lib, name)
        want = [ctypes.c_void_p if "*" in a else kinds[re.sub(r"\s*\w+$", "", a.strip())] for a in args.split(",")]
        assert want == _lib.LLM_SIGNATURES[name][1], name


def call(name, base, over):
    a = dict(base)
    a.update(over)
    assert set(a) == set(base), "a misspelled argument"
    return getattr(_lib.load(), name)(*a.values())


def refusals(name, base, cases):
    return [pytest.param(name, base, over, code, id=f"{name}:" + ",".join(f"{k}={v}" for k, v in over.items()))
            for code, group in cases.items() for over in group]


D, S = 64, 16
NORM = dict(Q=A, K=A + 0x1000, Qr=A + 0x2000, Kr=A + 0x3000, qw=A + 0x4000, kw=A + 0x5000, wtype=1, eps=1e-6,
            qb=4 * S * D, qh=S * D, qs=D, kb=2 * S * D, kh=S * D, ks=D, B=2, H=4, H_kv=2, S=S, D=D, dtype=0, rope=1,
            theta=1e4, table=TABLE, rows=S, positions=None, stream=None)
NORM_BAD = {
    INVALID: [dict(Q=None), dict(Qr=None), dict(K=None), dict(Kr=None), dict(Q=ODD), dict(Kr=ODD), dict(qw=ODD), dict(wtype=2),
              dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(qs=D + 4), dict(qb=-8), dict(kh=3), dict(ks=1 << 41),
              dict(B=0), dict(B=16385), dict(H=0), dict(H_kv=0), dict(H=16385), dict(S=0), dict(S=(1 << 20) + 1), dict(D=0),
              dict(D=63), dict(dtype=2), dict(rope=3), dict(theta=0.0), dict(theta=NAN), dict(table=None), dict(table=ODD),
              dict(rows=S - 1), dict(rows=(1 << 20) + 1), dict(positions=TABLE + 2), dict(table=A + 0x2000),
              dict(Qr=A + 0x1000), dict(Kr=A), dict(Qr=A + 0x3000), dict(Qr=A + 0x4000),
              dict(Qr=A, qs=4 * D, qh=D), dict(positions=A + 0x2000), dict(positions=A, rows=0)],
    UNSUPPORTED: [dict(D=96), dict(D=256), dict(D=96, rope=0, table=None), dict(D=96, K=None, Kr=None, H_kv=0),
                  dict(D=32, Qr=A, qs=32, qh=32 * S, qb=128 * S), dict(D=96, positions=TABLE + 4, rows=1),
                  dict(D=96, qb=0, qh=0, qs=0), dict(D=96, qw=None, kw=None)],
}
BWD = dict(Q=A, K=A + 0x1000, dQr=A + 0x2000, dKr=A + 0x3000, dQ=A + 0x4000, dK=A + 0x5000, dqw=A + 0x6000, dkw=A + 0x7000,
           qw=A + 0x8000, kw=A + 0x9000, wtype=1, eps=1e-6, qb=4 * S * D, qh=S * D, qs=D, kb=2 * S * D, kh=S * D, ks=D,
           dqb=4 * S * D, dqh=S * D, dqs=D, dkb=2 * S * D, dkh=S * D, dks=D, ws=A + 0xA000, wbytes=1 << 20, B=2, H=4, H_kv=2,
           S=S, D=D, dtype=0, rope=1, theta=1e4, table=TABLE, rows=S, positions=None, stream=None)
BWD_BAD = {
    INVALID: [dict(Q=None), dict(dQr=None), dict(dKr=None), dict(dQ=None), dict(dK=None), dict(dkw=None), dict(dqw=None),
              dict(ws=None), dict(ws=ODD), dict(wbytes=(2 + 1) * D * 4 - 1), dict(dQ=A), dict(dK=A + 0x3000),
              dict(dQ=A + 0x5000), dict(ws=A + 0x6000), dict(ws=TABLE), dict(dqs=D - 8), dict(dqh=0), dict(dkb=8),
              dict(qs=4), dict(dqs=D + 4), dict(eps=NAN), dict(wtype=-1), dict(H_kv=0), dict(rows=S - 1), dict(dqw=A + 0x6002)],
    UNSUPPORTED: [dict(D=96, dqs=96, dks=96), dict(D=96, dqs=96, K=None, dKr=None, dK=None, dkw=None),
                  dict(D=96, dqs=96, dks=96, dqw=None, dkw=None, ws=None, wbytes=0)],
}
APPEND = dict(Q=A, K=A + 0x1000, V=A + 0x2000, Qr=A + 0x3000, Kp=A + 0x4000, Vp=A + 0x5000, slots=A + 0x6000, qw=A + 0x7000,
              kw=A + 0x8000, wtype=1, norm=1, eps=1e-6, qt=4 * D, qh=D, kt=2 * D, kh=D, vt=2 * D, vh=D,
              kpp=2 * 16 * D, kph=16 * D, kps=D, vpp=2 * 16 * D, vph=16 * D, vps=D, T=3, H=4, H_kv=2, D=D, pages=8, page=16,
              dtype=0, rope=1, theta=1e4, table=TABLE, rows=5, positions=A + 0x9000, stream=None)
APPEND_BAD = {
    INVALID: [dict(Q=None), dict(K=None), dict(V=None), dict(Qr=None), dict(Kp=None), dict(Vp=None), dict(slots=None),
              dict(slots=A + 4), dict(Kp=ODD), dict(positions=None), dict(positions=A + 2), dict(norm=0), dict(eps=-1.0),
              dict(Kp=A + 0x5000), dict(Qr=A), dict(Vp=A + 0x2000), dict(qt=4), dict(kps=8), dict(vpp=0), dict(T=0),
              dict(T=(1 << 20) + 1), dict(H_kv=0), dict(pages=0), dict(page=0), dict(pages=1 << 27), dict(rows=0),
              dict(table=A + 0x4000), dict(rope=-1), dict(dtype=7)],
    UNSUPPORTED: [dict(page=8), dict(page=24), dict(page=1), dict(page=1 << 21, pages=1), dict(D=128 + 64, kps=192, kph=192,
                  kpp=192, vps=192, vph=192, vpp=192), dict(page=8, norm=0, qw=None, kw=None, eps=NAN),
                  dict(page=8, rope=0, positions=None, table=None)],
}

PAGED = dict(Q=A, Kp=A + 0x1000, Vp=A + 0x2000, table=A + 0x3000, lens=A + 0x4000, O=A + 0x5000, LSE=A + 0x6000,
             ws=A + 0x7000, wbytes=1 << 20, kpp=2 * 16 * D, kph=16 * D, kps=D, vpp=2 * 16 * D, vph=16 * D, vps=D, B=2, H=4,
             H_kv=2, D=D, pages=8, page=16, max_pages=4, rope=1, theta=1e4, rtable=TABLE, rows=64, mask=1, window=0, sinks=0,
             slopes=None, scale=0.125, stream=None)
PAGED_BAD = {
    INVALID: [dict(Q=None), dict(Kp=None), dict(Vp=None), dict(table=None), dict(O=None), dict(LSE=None), dict(ws=None),
              dict(Kp=ODD), dict(table=A + 0x3002), dict(lens=A + 1), dict(LSE=A + 2), dict(wbytes=1023), dict(O=A),
              dict(ws=A + 0x2000), dict(LSE=A + 0x4000), dict(ws=TABLE), dict(kps=D + 4), dict(vph=-8), dict(kps=1 << 25),
              dict(B=0), dict(H=3), dict(H_kv=0), dict(pages=0), dict(page=0), dict(max_pages=0),
              dict(max_pages=(1 << 16) + 1), dict(rows=63), dict(rtable=None), dict(theta=-1.0), dict(mask=3),
              dict(mask=2), dict(mask=2, window=-1), dict(sinks=1), dict(sinks=-1, mask=2, window=4), dict(scale=0.0),
              dict(scale=NAN), dict(rope=5)],
    UNSUPPORTED: [dict(page=8), dict(page=48), dict(D=96), dict(mask=2, window=4, sinks=1, slopes=A + 0x8000),
                  dict(D=96, lens=None, rope=0, rtable=None)],
}
STREAM = dict(Q=A, K=A + 0x1000, V=A + 0x2000, lens=A + 0x4000, O=A + 0x5000, LSE=A + 0x6000, ws=A + 0x7000, wbytes=1 << 20,
              B=2, H=4, H_kv=2, S_kv=100, D=D, rope=1, theta=1e4, rtable=TABLE, rows=100, window=10, sinks=2, scale=0.125,
              stream=None)
STREAM_BAD = {
    INVALID: [dict(Q=None), dict(K=ODD), dict(O=A + 0x1000), dict(ws=None), dict(wbytes=64), dict(S_kv=0),
              dict(S_kv=(1 << 20) + 1), dict(window=0), dict(sinks=0), dict(sinks=-2), dict(rows=99), dict(scale=INF)],
    UNSUPPORTED: [dict(D=96), dict(D=256, lens=None)],
}

FWD = dict(Q=A, K=A + 0x1000, V=A + 0x2000, O=A + 0x3000, LSE=A + 0x4000, ws=A + 0x5000, wbytes=2 * 2 * 100 * D * 2, B=2, H=4,
           H_kv=2, S=100, D=D, dtype=0, rope=1, theta=1e4, table=TABLE, rows=100, window=10, sinks=2, scale=0.125, stream=None)
FWD_BAD = {
    INVALID: [dict(Q=None), dict(LSE=None), dict(K=ODD), dict(O=A), dict(ws=None), dict(ws=ODD), dict(ws=A),
              dict(wbytes=2 * 2 * 100 * D * 2 - 1), dict(window=0), dict(sinks=0), dict(sinks=-1), dict(H_kv=3), dict(rows=99),
              dict(scale=-1.0), dict(S=0), dict(dtype=3), dict(rope=3)],
    UNSUPPORTED: [dict(D=96), dict(D=96, rope=0, ws=None, table=None), dict(D=96, dtype=1, ws=None, wbytes=0)],
}
GRAD = dict(Q=A, K=A + 0x1000, V=A + 0x2000, O=A + 0x3000, dO=A + 0x4000, LSE=A + 0x5000, dQ=A + 0x6000, dK=A + 0x7000,
            dV=A + 0x8000, ws=A + 0x9000, wbytes=1 << 24, B=2, H=4, H_kv=2, S=100, D=D, dtype=0, rope=1, theta=1e4, table=TABLE,
            rows=100, window=10, sinks=2, scale=0.125, stream=None)
GRAD_BAD = {
    INVALID: [dict(Q=None), dict(dO=None), dict(ws=None), dict(wbytes=0), dict(wbytes=1 << 12), dict(dK=A), dict(window=-3),
              dict(sinks=0), dict(rows=1), dict(dV=ODD)],
    UNSUPPORTED: [dict(D=96), dict(D=256, rope=0, table=None)],
}


@pytest.mark.parametrize("name,base,over,code", refusals("attnfuse_fwd_sinks", FWD, FWD_BAD)
                         + refusals("attnfuse_bwd_sinks", GRAD, GRAD_BAD)
                         + refusals("attnfuse_decode_paged", PAGED, PAGED_BAD)
                         + refusals("attnfuse_decode_sinks", STREAM, STREAM_BAD)
                         + refusals("attnfuse_qknorm_rope", NORM, NORM_BAD)
                         + refusals("attnfuse_qknorm_rope_bwd", BWD, BWD_BAD)
                         + refusals("attnfuse_qknorm_rope_append", APPEND, APPEND_BAD))
def test_refuses(name, base, over, code):
    assert call(name, base, over) == code


def test_qknorm_workspace_bytes():
    f = _lib.load().attnfuse_qknorm_rope_bwd_workspace_bytes
    assert f(2, 4, 2, 16, 64, 0) == (2 + 1) * 64 * 4          # two heads each; both batches in one workgroup's 64 rows
    assert f(2, 4, 2, 33, 64, 0) == (4 + 2) * 64 * 4          # a workgroup for each batch
    assert f(9, 4, 2, 16, 64, 0) == (6 + 3) * 64 * 4
    assert f(1, 32, 8, 8192, 128, 0) == 1024 * 128 * 4
    assert f(1, 1, 0, 1, 64, 1) == 64 * 4                     # no keys
    for bad in ((0, 1, 1, 1, 64, 0), (1, 1, 1, 0, 64, 0), (1, 1, 1, 1, 96, 0), (1, 1, 1, 1, 64, 2), (1, 1, -1, 1, 64, 0)):
        assert f(*bad) == 0


def test_decode_workspace_bytes():
    f = _lib.load().attnfuse_decode_paged_workspace_bytes
    assert f(1, 4, 2, 128, 64, 0, 0) == 256 + 4 * 64 * 4              # one part: four tiles
    assert f(1, 4, 2, 256, 64, 0, 0) == 256 + 4 * 2 * 64 * 4          # two, of four tiles each
    assert f(1, 4, 2, 1 << 20, 64, 32, 4) == 256 + 4 * 64 * 4         # a window's two tiles and the sinks'
    assert f(1, 4, 2, 1 << 20, 64, 193, 4) == 256 + 4 * 2 * 64 * 4    # its seven, and the sinks'
    for bad in ((0, 4, 2, 128, 64, 0, 0), (1, 3, 2, 128, 64, 0, 0), (1, 4, 2, 0, 64, 0, 0), (1, 4, 2, 128, 64, -1, 0),
                (1, 4, 2, 128, 64, 0, -1)):
        assert f(*bad) == 0


def test_sinks_workspace_bytes():
    lib = _lib.load()
    f = lib.attnfuse_fwd_sinks_workspace_bytes
    assert f(2, 2, 100, 64, 0, 1) == 2 * 2 * 100 * 64 * 2
    assert f(2, 2, 100, 64, 0, 0) == f(2, 2, 100, 64, 1, 1) == f(0, 2, 100, 64, 0, 1) == f(2, 2, 100, 96, 0, 1) == 0
    g, base = lib.attnfuse_bwd_sinks_workspace_bytes, lib.attnfuse_bwd_workspace_bytes
    # 32 sinks of 2 heads: a part for each four steps, of 2 query heads x 4 tiles
    # (without RoPE too Q and K pass through the workspace in fp16)
    assert g(1, 4, 2, 128, 64, 0, 10, 32) == g(1, 4, 2, 128, 64, 1, 10, 32) == base(1, 4, 2, 128, 64, 1) + 2 * 2 * 2 * 32 * 64 * 4
    assert g(1, 4, 2, 128, 64, 0, 100, 28) == base(1, 4, 2, 128, 64, 0)     # every key is visible
    for bad in ((0, 4, 2, 128, 64, 0, 10, 4), (1, 4, 2, 128, 64, 0, 0, 4), (1, 4, 2, 128, 64, 0, 10, 0), (1, 3, 2, 128, 64, 0, 10, 4)):
        assert g(*bad) == 0
