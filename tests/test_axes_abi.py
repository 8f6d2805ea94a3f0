"""Positions of several axes: the entry points reject bad arguments before any HIP call (CPU tests; no compute calls)."""
import ctypes

import pytest
import torch

from paper_2609_13612_amd import _lib, api
from test_llm_abi import APPEND, APPEND_BAD, BWD, BWD_BAD, INVALID, NORM, NORM_BAD, UNSUPPORTED, A, TABLE, call, refusals

D = NORM["D"]


def ints(*x):
    """A C array of ints that names itself by its values (the tests' names)."""
    return type("Ints", (ctypes.c_int * len(x),), {"__repr__": lambda self: "-".join(map(str, self))})(*x)


def with_axes(base, norm=True):
    """The arguments of a call at positions of one axis -> of three."""
    out = {}
    for k, v in base.items():
        if k == "stream":
            out.update(axes=3, sections=ints(10, 11, 11), order=0)
        if k == "eps" and norm:
            out["norm"] = 1
        out[k] = v
    out["positions"] = base["positions"] or TABLE + 0x1000
    return out


AXES_BAD = [dict(axes=0), dict(axes=5, sections=ints(6, 6, 6, 6, 8)), dict(sections=None), dict(sections=ints(10, 11, 12)),
            dict(sections=ints(0, 16, 16)), dict(sections=ints(-1, 17, 16)), dict(axes=2), dict(order=2), dict(order=-1),
            dict(rope=0), dict(positions=None), dict(positions=TABLE + 2), dict(table=None), dict(rows=0), dict(theta=0.0)]
FWD3, BWD3, APP3 = with_axes(NORM), with_axes(BWD), with_axes(APPEND, norm=False)


def usable(cases, base, drop=()):
    """The refusals of the calls at positions of one axis that mean the same here."""
    sized = ("D", "rows", "positions", "rope", "table")
    return {code: [over for over in group if not any(k in over for k in sized + drop)] for code, group in cases.items()}


@pytest.mark.parametrize("name,base,over,code", [
    *refusals("attnfuse_qknorm_axes", FWD3, {INVALID: AXES_BAD}), *refusals("attnfuse_qknorm_axes", FWD3, usable(NORM_BAD, FWD3)),
    *refusals("attnfuse_qknorm_axes", FWD3, {INVALID: [dict(norm=0), dict(norm=0, qw=None)],
                                             UNSUPPORTED: [dict(D=96, sections=ints(16, 16, 16)), dict(D=32, sections=ints(5, 5, 6))]}),
    *refusals("attnfuse_qknorm_axes_bwd", BWD3, {INVALID: AXES_BAD}), *refusals("attnfuse_qknorm_axes_bwd", BWD3, usable(BWD_BAD, BWD3)),
    *refusals("attnfuse_qknorm_axes_bwd", BWD3, {INVALID: [
        dict(norm=0), dict(norm=0, qw=None, kw=None), dict(norm=0, qw=None, kw=None, dqw=None),
        dict(norm=0, qw=None, kw=None, dqw=None, dkw=None, dQ=None),
        dict(norm=0, qw=None, kw=None, dqw=None, dkw=None, dQ=A + 0x2000),
        dict(norm=0, qw=None, kw=None, dqw=None, dkw=None, dKr=None),
        dict(norm=0, qw=None, kw=None, dqw=None, dkw=None, dqs=D - 8),
        dict(norm=0, qw=None, kw=None, dqw=None, dkw=None, dQ=TABLE),
        dict(norm=0, qw=None, kw=None, dqw=None, dkw=None, rope=0),
        dict(norm=0, qw=None, kw=None, dqw=None, dkw=None, positions=None)]}),
    *refusals("attnfuse_qknorm_axes_append", APP3, {INVALID: AXES_BAD}),
    *refusals("attnfuse_qknorm_axes_append", APP3, usable(APPEND_BAD, APP3)),
])
def test_refused(name, base, over, code):
    assert call(name, base, over) == code


FILL = dict(table=TABLE, rows=8, D=64, theta=1e4, axes=2, sections=ints(16, 16), order=0, frequencies=1, stream=None)


@pytest.mark.parametrize("name,base,over,code", refusals("attnfuse_axes_table_fill", FILL, {
    INVALID: [dict(table=None), dict(table=TABLE + 8), dict(rows=0), dict(rows=(1 << 20) + 1), dict(theta=-1.0), dict(axes=3),
              dict(sections=ints(16, 15)), dict(order=3), dict(frequencies=2), dict(D=63)],
    UNSUPPORTED: [dict(D=96, sections=ints(24, 24))]}))
def test_table_refused(name, base, over, code):
    assert call(name, base, over) == code


def test_python_refuses():
    """What Python checks itself, before it needs a GPU."""
    pos = torch.zeros(2, 1, 4, dtype=torch.int32)
    good = ((16, 16), "blocks", "shared", True, "neox", 64, pos)
    assert api._axes(*good) == ((16, 16), "blocks")
    assert api._axes(None, "blocks", "shared", True, "none", 64, None) is None
    for i, bad in ((0, None), (0, (16, 17)), (0, (32, 0)), (0, ()), (0, (4, 4, 8, 8, 8)), (1, "rows"), (2, "mine"), (4, "none"), (6, None)):
        args = list(good)
        args[i] = bad
        if bad is None and i == 0:
            args[3] = False   # without sections there is always a norm
        with pytest.raises(ValueError):
            api._axes(*args)
    q = torch.zeros(1, 2, 4, 64)
    for f in (api.attnfuse_qknorm_rope, api.attnfuse_qknorm_rope_append, api.attnfuse_qknorm_rope_bwd):
        with pytest.raises(ValueError, match="GPU"):
            f(*([q] * (6 if f is api.attnfuse_qknorm_rope_append else 4)), sections=(16, 16), positions=pos, max_positions=4)
    assert "attnfuse_qknorm_axes" in _lib.LLM_SIGNATURES


def test_sections_are_whole_numbers():
    pos = torch.zeros(2, 1, 4, dtype=torch.int32)
    assert api._axes((16.0, 16), "blocks", "shared", True, "neox", 64, pos) == ((16, 16), "blocks")
    with pytest.raises(ValueError, match="whole"):
        api._axes((16.5, 16.5), "blocks", "shared", True, "neox", 64, pos)   # (not taken as 16, 16)


@pytest.mark.parametrize("bad", [dict(sections=(16.5, 16.5)), dict(sections=(16, 17)), dict(sections=()),
                                 dict(sections=(16, 16), section_order="rows"), dict(sections=(16, 16), frequencies="mine")], ids=str)
def test_a_table_checks_its_sections_as_the_calls_do(bad):
    with pytest.raises(ValueError, match="section"):
        api.rope_table(64, 1e4, 8, "cuda:0", **bad)
