"""New tokens over pages: the entry point rejects bad arguments before any HIP call (CPU tests; no compute calls)."""
import pytest
import torch

from paper_2609_13612_amd import _lib, api
from test_llm_abi import INVALID, NAN, ODD, UNSUPPORTED, A, call, refusals

D = 64
PAGED = dict(Q=A, Kp=A + 0x1000, Vp=A + 0x2000, table=A + 0x3000, starts=A + 0x4000, lens=A + 0x5000, prefix=A + 0x6000,
             plen=A + 0x7000, O=A + 0x8000, LSE=A + 0x9000, ws=A + 0xA000, wbytes=1 << 40, kpp=2 * 16 * D, kph=16 * D, kps=D,
             vpp=2 * 16 * D, vph=16 * D, vps=D, T=5, B=3, H=4, H_kv=2, D=D, pages=8, page=16, most=4, ahead=2, scale=0.125,
             stream=None)
BAD = {
    INVALID: [dict(Q=None), dict(Kp=None), dict(Vp=None), dict(table=None), dict(O=None), dict(LSE=None), dict(ws=None),
              dict(Q=ODD), dict(Vp=ODD), dict(O=ODD), dict(ws=ODD), dict(table=A + 2), dict(starts=A + 1), dict(lens=A + 2),
              dict(prefix=A + 2), dict(plen=A + 2), dict(LSE=A + 2), dict(starts=None), dict(prefix=None), dict(ahead=0),
              dict(ahead=0, prefix=None), dict(ahead=-1), dict(wbytes=0), dict(O=A), dict(LSE=A + 0x5000), dict(O=A + 0x1000),
              dict(O=A + 0xA000), dict(LSE=A + 0x8000), dict(ws=A + 0x6000), dict(ws=A + 0x7000), dict(T=0), dict(B=0), dict(H=0),
              dict(H_kv=0), dict(H_kv=3), dict(H=16385, H_kv=1), dict(B=1 << 16), dict(T=(1 << 20) + 1), dict(D=63), dict(pages=0),
              dict(page=0), dict(most=0), dict(most=(1 << 16) + 1), dict(ahead=(1 << 16) + 1), dict(kps=4), dict(vph=-8),
              dict(kpp=1 << 41), dict(vps=(1 << 24) + 8), dict(scale=0.0), dict(scale=NAN), dict(scale=-1.0),
              dict(T=1 << 20, H=2048, H_kv=2048)],
    UNSUPPORTED: [dict(D=96), dict(page=24), dict(page=8), dict(page=48)],
}


@pytest.mark.parametrize("name,base,over,code", refusals("attnfuse_fwd_paged", PAGED, BAD))
def test_refused(name, base, over, code):
    assert call(name, base, over) == code


def test_one_token_each_needs_as_many_sequences():
    assert call("attnfuse_fwd_paged", PAGED, dict(starts=None, T=4)) == INVALID


def test_workspace_bytes():
    f = _lib.load().attnfuse_fwd_paged_workspace_bytes
    for bad in ((0, 1, 4, 2, 64, 64, 0), (4, 0, 4, 2, 64, 64, 0), (4, 1, 4, 3, 64, 64, 0), (4, 1, 4, 2, 63, 64, 0), (4, 1, 4, 2, 64, 0, 0),
                (4, 1, 4, 2, 64, 64, -1), (4, 1, 4, 2, 64, (1 << 20) + 1, 0), (1 << 20, 1, 4096, 1, 64, 64, 0)):
        assert f(*bad) == 0
    # partials of (max, sum, D values) of every (token, head), whole numbers of them
    for T, B, H, Hkv, own, ahead in ((4, 4, 32, 8, 64, 512), (32, 32, 32, 8, 1024, 32768), (50, 3, 12, 12, 320, 5008)):
        n = f(T, B, H, Hkv, 128, own, ahead)
        parts = n // (T * H * (128 + 2) * 4)
        assert parts >= 2 and n - parts * T * H * (128 + 2) * 4 < 512
    assert f(65535, 65535, 64, 64, 128, 64, 64) > 0 and f(1 << 20, 1, 1024, 8, 128, 1 << 20, 0) == 0   # (results are written at once)
    assert f(1 << 20, 65535, 1024, 1024, 128, 64, 0) == 0 and f(1 << 20, 4, 1024, 1, 128, 64, 1 << 20) == 0
    assert api.attnfuse_fwd_paged_workspace_bytes(4, 4, 32, 8, 128, 64, 512) == f(4, 4, 32, 8, 128, 64, 512)


def test_python_refuses():
    q, kv, table = torch.zeros(2, 4, 64), torch.zeros(3, 2, 16, 64), torch.zeros(2, 1, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        api.attnfuse_fwd_paged(q, kv, kv, table, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="q_starts"):
        api.attnfuse_fwd_paged(q, kv, kv, table, None)
    with pytest.raises(ValueError, match="prefix_table"):
        api.attnfuse_decode_paged(q, kv, kv, table, prefix_len=table[0])
    with pytest.raises(ValueError, match="rotated"):
        api.attnfuse_decode_paged(q, kv, kv, table, prefix_table=table[0], rope="neox")


# A launch has fewer than 2^32 threads: fewer than 2^24 workgroups of 256, or 2^23 of 512, and as many rows of partials to join
# as 2^32 threads have, D / 4 a row.
TOO_MANY = [
    dict(T=65535, B=65535, H=512, H_kv=512),                                # a workgroup for each sequence and K/V head
    dict(T=65535, B=65535, H=512, H_kv=512, starts=None),
    dict(T=65535, B=65535, H=512, H_kv=512, ahead=0, prefix=None, plen=None),
    dict(T=1 << 20, B=65535, H=128, H_kv=8, D=128, kps=128, vps=128),       # 2^27 rows of at least two partials
    dict(T=1 << 20, B=65535, H=256, H_kv=8, D=64),
]


@pytest.mark.parametrize("over", TOO_MANY, ids=str)
def test_what_cannot_be_launched_is_refused(over):
    assert call("attnfuse_fwd_paged", PAGED, over) == INVALID
    a = {**PAGED, **over}
    assert _lib.load().attnfuse_fwd_paged_workspace_bytes(a["T"], a["B"], a["H"], a["H_kv"], a["D"], a["most"] * a["page"],
                                                          a["ahead"] * a["page"]) == 0


def test_the_largest_launches_are_not_refused():
    f = _lib.load().attnfuse_fwd_paged_workspace_bytes
    assert f((1 << 20) - 1, 65535, 128, 8, 128, 64, 32) > 0 and f((1 << 20) - 1, 65535, 256, 8, 64, 64, 32) > 0
    assert f(65535, 65535, 250, 250, 128, 64, 32) > 0    # (four waves: eight would be too many threads)
