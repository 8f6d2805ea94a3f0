"""Norm and rotation at positions of several axes, its backward, and the form that writes new tokens to pages, against the
definition in 64 bits.

Tolerances are those of the same kernels at positions of one axis (test_gpu_qknorm.py): the output rounded once, before it
under 64 u (u = 2^-24) of a row's largest |w x r| (without a norm of its largest |x|: a rotation alone has two products with
rounded cos and sin and their sum, under 8 u), 128 u in the gradient, (rows of a thread + 148) u in a weight's.
"""
import pytest
import torch

from axes_ref import axes_bwd, axes_fwd
from gpu_util import announce, need_gpu
from llm_ref import U32, assert_within, half_step
from paper_2609_13612_amd import api, autograd

pytestmark = pytest.mark.gpu
EPS = 1e-6
MOST = 5000


def rows(shape, dtype, g, layout):
    """[B, H, S, D] of N(0, 1), contiguous ("bhsd"), positions first ("bshd") or a slice of a wider projection ("slice")."""
    B, H, S, D = shape
    if layout == "bhsd":
        return torch.randn(shape, generator=g).to(dtype).cuda()
    wide = torch.randn(B, S, H + (3 if layout == "slice" else 0), D, generator=g).to(dtype).cuda()
    return wide[:, :, 1:1 + H].transpose(1, 2) if layout == "slice" else wide.transpose(1, 2)


def weights(D, kind, dtype, g):
    if kind == "none":
        return None, None
    return tuple((1 + 0.2 * torch.randn(D, generator=g)).to(torch.float32 if kind == "fp32" else dtype).cuda() for _ in "qk")


def cfg_of(rope, theta, sections, order, ladder, norm, pos):
    return dict(eps=EPS, rope=rope, theta=theta, sections=sections, section_order=order, frequencies=ladder, norm=norm,
                positions=pos, max_positions=MOST)


def positions(axes, lead, g):
    return torch.randint(0, MOST, (axes, *lead), generator=g, dtype=torch.int32)


BF, F32 = torch.bfloat16, torch.float32
CASES = [
    # B, H, Hkv, S, D, dtype, rope, layout, weights, sections, order, frequencies, norm
    (1, 32, 8, 300, 128, BF, "neox", "slice", "rows", (16, 24, 24), "blocks", "shared", True),
    (2, 12, 12, 77, 64, BF, "interleaved", "bshd", "fp32", (16, 16), "blocks", "own", True),
    (3, 5, 2, 33, 128, F32, "neox", "bhsd", "fp32", (24, 20, 20), "turns", "shared", True),
    (1, 1, 1, 1, 64, BF, "neox", "bhsd", "rows", (10, 11, 11), "turns", "own", True),
    (2, 7, 3, 1, 128, F32, "interleaved", "slice", "none", (7, 28, 29), "turns", "shared", True),
    (1, 3, 1, 2049, 64, F32, "interleaved", "bshd", "none", (1, 31), "blocks", "own", False),
    (2, 6, 0, 40, 128, BF, "interleaved", "slice", "rows", (1, 62, 1), "blocks", "shared", True),      # no keys
    (2, 6, 0, 40, 64, BF, "neox", "slice", "none", (5, 27), "turns", "shared", False),
    (4, 16, 4, 1000, 128, BF, "neox", "bhsd", "none", (16, 16, 16, 16), "turns", "shared", False),
    (1, 64, 8, 700, 64, BF, "neox", "slice", "rows", (8, 8, 8, 8), "blocks", "own", True),              # more units than workgroups
    (67, 5, 2, 1, 128, BF, "neox", "slice", "fp32", (32, 32), "turns", "own", True),                    # several sequences a workgroup
    (23, 6, 3, 3, 64, BF, "interleaved", "bhsd", "none", (9, 10, 13), "blocks", "shared", False),
    (5, 4, 4, 16, 128, F32, "neox", "bshd", "rows", (64,), "blocks", "shared", True),
    (2, 9, 3, 2000, 128, F32, "neox", "slice", "fp32", (31, 2, 31), "blocks", "shared", True),
    (12, 7, 3, 900, 64, BF, "interleaved", "bshd", "none", (3, 29), "turns", "own", False),
]


@pytest.mark.parametrize("B,H,Hkv,S,D,dtype,rope,layout,wkind,sections,order,ladder,norm", CASES,
                         ids=lambda x: str(x).replace("torch.", "").replace(" ", ""))
def test_forward_and_backward(B, H, Hkv, S, D, dtype, rope, layout, wkind, sections, order, ladder, norm):
    need_gpu()
    announce(f"axes B={B} H={H}/{Hkv} S={S} D={D} {dtype} {rope} {layout} {wkind} {sections} {order} {ladder} {norm}")
    g = torch.Generator().manual_seed(S + D)
    q, k = rows((B, H, S, D), dtype, g, layout), rows((B, Hkv, S, D), dtype, g, layout) if Hkv else None
    qw, kw = weights(D, wkind, dtype, g)
    kw = kw if Hkv else None
    do = [rows((B, h, S, D), dtype, g, "bhsd") for h in (H, Hkv) if h]
    pos = positions(len(sections), (B, S), g)
    at = pos[:, :, None]
    cfg = cfg_of(rope, 500000.0, sections, order, ladder, norm, pos.cuda())
    variant = (rope, 500000.0, sections, order, ladder)
    out = api.attnfuse_qknorm_rope(q, k, qw, kw, **cfg)
    args = (q, k) if norm else (None, None)
    grads = api.attnfuse_qknorm_rope_bwd(*args, do[0], do[1] if Hkv else None, qw, kw, **cfg)
    assert (out[1] is None and grads[1] is None) == (not Hkv)
    before, after = (64, 128) if norm else (8, 8)
    for i, (x, w) in enumerate(((q, qw), (k, kw))[: len(do)]):
        want, size = axes_fwd(x, w, at, variant, norm, EPS)
        assert out[i].is_contiguous() and out[i].dtype == dtype
        assert_within(out[i], want, half_step(dtype) * want.abs() + before * U32 * size, "qk"[i] + "'")
        dx, dw, dsize, wsize = axes_bwd(x, w, do[i], at, variant, norm, EPS)
        assert_within(grads[i], dx, half_step(dtype) * dx.abs() + after * U32 * dsize, "d" + "qk"[i])
        if not norm:
            assert grads[2] is None and grads[3] is None
            continue
        wt = torch.float32 if wkind in ("fp32", "none") else dtype
        n = B * x.shape[1] * S
        assert_within(grads[2 + i], dw, half_step(wt) * dw.abs() + (n / 32 + 148) * U32 * wsize, "dw of " + "qk"[i])
    again = api.attnfuse_qknorm_rope_bwd(*args, do[0], do[1] if Hkv else None, qw, kw, **cfg)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(again, grads)), "another call, other bits"


@pytest.mark.parametrize("rope", ["neox", "interleaved"])
@pytest.mark.parametrize("D", [64, 128])
def test_one_axis_and_equal_axes_are_the_plain_rotation(D, rope):
    """The same table, the same arithmetic: the same bits."""
    need_gpu()
    announce(f"axes as one, D={D} {rope}")
    g = torch.Generator().manual_seed(D)
    q, k = rows((2, 8, 40, D), BF, g, "slice"), rows((2, 2, 40, D), BF, g, "slice")
    qw, kw = weights(D, "rows", BF, g)
    dq, dk = rows((2, 8, 40, D), BF, g, "bhsd"), rows((2, 2, 40, D), BF, g, "bhsd")
    pos = positions(1, (2, 40), g).cuda()
    plain = dict(eps=EPS, rope=rope, theta=10000.0, positions=pos[0], max_positions=MOST)
    want = api.attnfuse_qknorm_rope(q, k, qw, kw, **plain) + api.attnfuse_qknorm_rope_bwd(q, k, dq, dk, qw, kw, **plain)
    for sections, order, p in (((D // 2,), "blocks", pos), ((D // 4, D // 4 - 3, 3), "turns", pos.expand(3, 2, 40).contiguous())):
        cfg = cfg_of(rope, 10000.0, sections, order, "shared", True, p)
        got = api.attnfuse_qknorm_rope(q, k, qw, kw, **cfg) + api.attnfuse_qknorm_rope_bwd(q, k, dq, dk, qw, kw, **cfg)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("norm", [True, False])
def test_against_differences(norm):
    """The gradients of a random projection of the outputs against central differences of the definition in 64 bits."""
    need_gpu()
    announce(f"axes differences, norm {norm}")
    g = torch.Generator().manual_seed(5)
    q, do = torch.randn(1, 2, 3, 64, generator=g), torch.randn(1, 2, 3, 64, generator=g)
    w = 1 + 0.2 * torch.randn(64, generator=g) if norm else None
    pos = positions(3, (1, 3), g)
    variant = ("neox", 10000.0, (10, 11, 11), "turns", "own")
    cfg = cfg_of(*variant, norm, pos.cuda())
    dq, _, dw, _ = api.attnfuse_qknorm_rope_bwd(q.cuda(), None, do.cuda(), None, w.cuda() if norm else None, **cfg)

    def loss(x, w):
        return (axes_fwd(x, w, pos[:, :, None], variant, norm, EPS)[0] * do.double()).sum()

    h = 1e-5
    for _ in range(40):
        i = int(torch.randint(q.numel(), (1,), generator=g))
        e = torch.zeros(q.numel(), dtype=torch.float64)
        e[i] = h
        diff = (loss(q.double() + e.view(q.shape), w) - loss(q.double() - e.view(q.shape), w)) / (2 * h)
        assert abs(float(dq.flatten()[i]) - diff) < 2e-5   # fp32: 128 u of about 8; differences: h^2 and 2^-53 / h
        if norm:
            e = torch.zeros(64, dtype=torch.float64)
            e[i % 64] = h
            diff = (loss(q, w.double() + e) - loss(q, w.double() - e)) / (2 * h)
            assert abs(float(dw[i % 64]) - diff) < 2e-5


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("keys", [True, False])
@pytest.mark.parametrize("norm", [True, False])
def test_autograd(monkeypatch, norm, keys, native):
    """The differentiable call gives the outputs and gradients of the direct ones, also where one output is not used, keeps
    its gradients under create_graph, and refuses a second derivative."""
    need_gpu()
    announce(f"axes autograd norm={norm} keys={keys} native={native}")
    if not native:
        monkeypatch.setattr(api, "_native", None)
    else:
        assert api._native is not None
    g = torch.Generator().manual_seed(6)
    q, k = (rows((2, h, 50, 128), BF, g, "slice").detach().requires_grad_() for h in (8, 2))
    qw, kw = (w.requires_grad_() for w in weights(128, "rows", BF, g)) if norm else (None, None)
    do, dk = rows((2, 8, 50, 128), BF, g, "bhsd"), rows((2, 2, 50, 128), BF, g, "bhsd")
    cfg = cfg_of("neox", 10000.0, (16, 24, 24), "blocks", "own", norm, positions(3, (2, 50), g).cuda())
    leaves = [t for t in ((q, k, qw, kw) if keys else (q, qw)) if t is not None]
    ins = (q, k, qw, kw) if keys else (q, None, qw, None)
    outs = autograd.qknorm_rope(*ins, **cfg)
    outs = outs if keys else (outs,)
    want = api.attnfuse_qknorm_rope(*(None if t is None else t.detach() for t in ins), **cfg)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    grads = torch.autograd.grad(outs, leaves, (do, dk) if keys else (do,), retain_graph=True)
    direct = api.attnfuse_qknorm_rope_bwd(ins[0], ins[1], do, dk if keys else None, qw, ins[3], **cfg)
    assert all(torch.equal(a, b) for a, b in zip(grads, [x for x in direct if x is not None]))
    if keys:   # the other output counts with a gradient of 0
        alone = torch.autograd.grad(outs[0], (q, k), do, retain_graph=True)
        assert torch.equal(alone[0], grads[0]) and not alone[1].any()
    do = do.clone().requires_grad_()
    twice = torch.autograd.grad(outs, leaves, (do, dk) if keys else (do,), create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(twice, grads))
    with pytest.raises(RuntimeError, match="twice"):
        twice[0].float().square().sum().backward()


@pytest.mark.parametrize("native", [True, False])
def test_positions_out_of_range_give_nan(monkeypatch, native):
    """One axis out of range makes the row NaN, whatever longer table there is; every other row is what it was."""
    need_gpu()
    announce(f"axes out of range, native={native}")
    if not native:
        monkeypatch.setattr(api, "_native", None)
    g = torch.Generator().manual_seed(7)
    q, pos = rows((1, 3, 9, 64), BF, g, "bhsd"), positions(2, (1, 9), g)
    for norm in (True, False):
        cfg = cfg_of("neox", 10000.0, (16, 16), "blocks", "shared", norm, pos.cuda())
        want = api.attnfuse_qknorm_rope(q, **cfg)[0]
        bad = pos.clone()
        bad[0, 0, 2], bad[1, 0, 5], bad[1, 0, 7] = MOST, -1, 2 ** 31 - 1
        cfg["positions"] = bad.cuda()
        got = api.attnfuse_qknorm_rope(q, **cfg)[0]
        grad = api.attnfuse_qknorm_rope_bwd(q, None, q, None, **cfg)[0]
        hit = torch.zeros(9, dtype=torch.bool)
        hit[[2, 5, 7]] = True
        assert got[0, :, hit].isnan().all() and grad[0, :, hit].isnan().all()
        assert torch.equal(got[0, :, ~hit], want[0, :, ~hit]) and grad[0, :, ~hit].isfinite().all()


APPEND = [
    # T, H, Hkv, D, page, dtype, rope, weights, norm, sections, order, frequencies, pages' layout
    (1, 32, 8, 128, 16, BF, "neox", "rows", True, (16, 24, 24), "blocks", "shared", "phsd"),
    (37, 12, 12, 64, 32, BF, "interleaved", "none", False, (16, 16), "turns", "own", "pshd"),
    (700, 9, 3, 128, 16, BF, "neox", "fp32", True, (7, 28, 29), "turns", "shared", "pshd"),
    (5, 4, 1, 64, 256, F32, "interleaved", "none", True, (8, 8, 8, 8), "blocks", "own", "phsd"),
    (2500, 64, 8, 128, 64, BF, "neox", "none", False, (24, 20, 20), "turns", "shared", "phsd"),
]


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("T,H,Hkv,D,page,dtype,rope,wkind,norm,sections,order,ladder,layout", APPEND,
                         ids=lambda x: str(x).replace("torch.", "").replace(" ", ""))
def test_append(monkeypatch, T, H, Hkv, D, page, dtype, rope, wkind, norm, sections, order, ladder, layout, native):
    need_gpu()
    announce(f"axes append T={T} H={H}/{Hkv} D={D} page={page} {dtype} {rope} {wkind} {norm} {sections} {order} {ladder} {layout}")
    if not native:
        monkeypatch.setattr(api, "_native", None)
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, H + 2 * Hkv, D, generator=g).to(dtype).cuda()
    q, k, v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    pages = 2 * (T // page) + 3
    shape = (pages, Hkv, page, D) if layout == "phsd" else (pages, page, Hkv, D)
    kc, vc = (torch.randn(shape, generator=g).to(dtype).cuda() for _ in "kv")
    kc, vc = (kc, vc) if layout == "phsd" else (kc.transpose(1, 2), vc.transpose(1, 2))
    slots = torch.randperm(pages * page, generator=g)[:T]
    slots[T // 2:T // 2 + T // 7] = -1
    if T > 4:
        slots[1] = pages * page   # behind the last page
    kept = (slots >= 0) & (slots < pages * page)
    qw, kw = weights(D, wkind, dtype, g)
    pos = positions(len(sections), (T,), g)
    cfg = cfg_of(rope, 10000.0, sections, order, ladder, norm, pos.cuda())
    k0, v0 = kc.clone(), vc.clone()
    qr = api.attnfuse_qknorm_rope_append(q, k, v, kc, vc, slots.cuda(), qw, kw, **cfg)
    before = 64 if norm else 8
    variant = (rope, 10000.0, sections, order, ladder)
    want, size = axes_fwd(q, qw, pos[:, :, None], variant, norm, EPS)
    assert_within(qr, want, half_step(dtype) * want.abs() + before * U32 * size, "q'")
    want, size = axes_fwd(k, kw, pos[:, :, None], variant, norm, EPS)
    at = slots[kept]
    got = kc.transpose(1, 2).reshape(pages * page, Hkv, D)
    assert_within(got[at.cuda()], want[kept], half_step(dtype) * want[kept].abs() + before * U32 * size[kept], "k'")
    others = torch.ones(pages * page, dtype=torch.bool)
    others[at] = False
    assert torch.equal(got[others.cuda()], k0.transpose(1, 2).reshape(pages * page, Hkv, D)[others.cuda()])
    v0.transpose(1, 2)[at.cuda() // page, at.cuda() % page] = v[kept.cuda()]
    assert torch.equal(vc, v0)


@pytest.mark.parametrize("T", [2, 90])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("order", ["blocks", "turns"])
@pytest.mark.parametrize("rope", ["neox", "interleaved"])
@pytest.mark.parametrize("D,sections", [(64, (16, 16)), (64, (5, 27)), (64, (8, 12, 12)), (64, (8, 8, 8, 8)), (128, (32, 32)),
                                        (128, (7, 28, 29)), (128, (16, 16, 16, 16))], ids=lambda x: str(x).replace(" ", ""))
def test_append_every_pair(monkeypatch, D, sections, rope, order, dtype, T):
    """Every pair turns by its own axis's position, in the head sizes, orders and types of the append."""
    test_append(monkeypatch, T, 12, 4, D, 32, dtype, rope, "rows", True, sections, order, "own", "phsd", True)


@pytest.mark.parametrize("norm", [True, False])
def test_native_and_python_marshalling_agree(monkeypatch, norm):
    need_gpu()
    announce(f"axes marshalling, norm {norm}")
    assert api._native is not None, "the native binding is not built"
    g = torch.Generator().manual_seed(9)
    q, k = rows((2, 8, 30, 64), BF, g, "slice"), rows((2, 4, 30, 64), BF, g, "slice")
    qw, kw = weights(64, "rows", BF, g) if norm else (None, None)
    dq, dk = rows((2, 8, 30, 64), BF, g, "bhsd"), rows((2, 4, 30, 64), BF, g, "bhsd")
    cfg = cfg_of("interleaved", 10000.0, (10, 11, 11), "turns", "own", norm, positions(3, (2, 30), g).cuda())
    taken, real = [], api._native

    class Spy:
        def __getattr__(self, name):
            def call(*args):
                r = getattr(real, name)(*args)
                taken.append((name, r is not None))
                return r
            return call

    def calls():
        return api.attnfuse_qknorm_rope(q, k, qw, kw, **cfg) + api.attnfuse_qknorm_rope_bwd(q, k, dq, dk, qw, kw, **cfg)

    calls()   # (builds the table)
    monkeypatch.setattr(api, "_native", Spy())
    a = calls()
    assert taken == [("axes", True), ("axes_bwd", True)]
    monkeypatch.setattr(api, "_native", None)
    b = calls()
    assert all(x is y is None or (torch.equal(x, y) and x.stride() == y.stride()) for x, y in zip(a, b))


@pytest.mark.parametrize("native", [True, False])
def test_refusals(monkeypatch, native):
    need_gpu()
    announce(f"axes refusals native={native}")
    if not native:
        monkeypatch.setattr(api, "_native", None)
    g = torch.Generator().manual_seed(10)
    q, pos = rows((1, 4, 9, 64), BF, g, "bhsd"), positions(2, (1, 9), g).cuda()
    good = cfg_of("neox", 10000.0, (16, 16), "blocks", "own", True, pos)
    w = torch.ones(64, device="cuda")
    api.attnfuse_qknorm_rope(q, None, w, **good)
    for bad in (dict(sections=(16, 17)), dict(sections=(32, 0)), dict(sections=(8, 8, 16)), dict(sections=()), dict(rope="none"),
                dict(section_order="rows"), dict(frequencies="mine"), dict(positions=None), dict(positions=pos[0]),
                dict(positions=pos.long()), dict(positions=pos.cpu()), dict(max_positions=None), dict(max_positions=0),
                dict(norm=False), dict(sections=None, norm=False)):
        with pytest.raises((ValueError, TypeError)):
            api.attnfuse_qknorm_rope(q, None, w, **{**good, **bad})
        with pytest.raises((ValueError, TypeError)):
            autograd.qknorm_rope(q, None, w, **{**good, **bad})
    table = api.rope_table(64, 10000.0, 100, sections=(16, 16), frequencies="own")
    with pytest.raises(ValueError):   # a table of fewer rows than max_positions
        api.attnfuse_qknorm_rope(q, None, w, **good, rope_table=table)
    with pytest.raises(api.AttnFuseError):
        api.attnfuse_qknorm_rope(q[..., :32].contiguous(), None, **{**good, "sections": (8, 8)})   # no kernel for D = 32


def test_a_given_table_is_used_to_its_rows():
    """rope_table without max_positions: positions below its rows, others NaN; the bits of the binding's own table."""
    need_gpu()
    announce("axes given table")
    g = torch.Generator().manual_seed(14)
    q, pos = rows((1, 4, 9, 128), BF, g, "bhsd"), positions(3, (1, 9), g) % 100
    pos[1, 0, 4] = 100
    table = api.rope_table(128, 10000.0, 100, sections=(24, 20, 20), section_order="turns", frequencies="own")
    cfg = cfg_of("neox", 10000.0, (24, 20, 20), "turns", "own", False, pos.cuda())
    want = api.attnfuse_qknorm_rope(q, **cfg)[0]
    got = api.attnfuse_qknorm_rope(q, **{**cfg, "max_positions": None}, rope_table=table)[0]
    hit = torch.arange(9) == 4
    assert got[:, :, hit].isnan().all() and torch.equal(got[:, :, ~hit], want[:, :, ~hit])


def test_captured_step_replays():
    """A training step captured into a graph (leaves of its own, a cold table) and replayed on new inputs."""
    need_gpu()
    announce("axes graph")
    g = torch.Generator().manual_seed(11)
    q, k = (rows((1, h, 70, 128), BF, g, "bhsd").requires_grad_() for h in (8, 2))
    w = (1 + 0.2 * torch.randn(128, generator=g)).cuda().requires_grad_()
    pos = positions(3, (1, 70), g).cuda()
    do, dk = rows((1, 8, 70, 128), BF, g, "bhsd"), rows((1, 2, 70, 128), BF, g, "bhsd")
    cfg = cfg_of("neox", 70000.0, (16, 24, 24), "turns", "own", True, pos)

    def step():
        outs = autograd.qknorm_rope(q, k, w, w, **cfg)
        return (*outs, *torch.autograd.grad(outs, (q, k, w), (do, dk)))

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for i in range(3):
        with torch.no_grad():
            for t in (q, k, do, dk):
                t.copy_(torch.randn(t.shape, generator=g).to(t.dtype).cuda())
            pos.copy_(torch.randint(0, MOST, pos.shape, generator=g, dtype=torch.int32).cuda())
        graph.replay()
        torch.cuda.synchronize()
        mine = [x.detach().clone() for x in (q, k, w)]
        other = dict(cfg, positions=pos.clone())
        outs = api.attnfuse_qknorm_rope(mine[0], mine[1], mine[2], mine[2], **other)
        grads = api.attnfuse_qknorm_rope_bwd(mine[0], mine[1], do, dk, mine[2], mine[2], **other)
        want = (*outs, grads[0], grads[1], grads[2] + grads[3])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), f"replay {i}"


def test_longest_sequence():
    """S = 2^20: sampled rows against the definition, forward and backward."""
    need_gpu()
    announce("axes S=2^20")
    g = torch.Generator().manual_seed(18)
    S, variant = 1 << 20, ("neox", 500000.0, (10, 11, 11), "turns", "shared")
    q, w = rows((1, 2, S, 64), BF, g, "bshd"), weights(64, "rows", BF, g)[0]
    do, pos = rows((1, 2, S, 64), BF, g, "bhsd"), positions(3, (1, S), g)
    cfg = cfg_of(*variant, True, pos.cuda())
    out = api.attnfuse_qknorm_rope(q, None, w, **cfg)[0]
    dq = api.attnfuse_qknorm_rope_bwd(q, None, do, None, w, **cfg)[0]
    at = torch.cat((torch.arange(5), torch.randint(0, S, (300,), generator=g), torch.arange(S - 5, S)))
    take = lambda t: t[:, :, at.cuda()].cpu()   # noqa: E731
    want, size = axes_fwd(take(q), w, pos[:, :, None][..., at], variant, True, EPS)
    assert_within(take(out), want, half_step(BF) * want.abs() + 64 * U32 * size, "q'")
    dx, _, dsize, _ = axes_bwd(take(q), w, take(do), pos[:, :, None][..., at], variant, True, EPS)
    assert_within(take(dq), dx, half_step(BF) * dx.abs() + 128 * U32 * dsize, "dq")


def test_on_another_stream():
    need_gpu()
    announce("axes stream")
    g = torch.Generator().manual_seed(12)
    q = rows((1, 16, 4000, 128), BF, g, "bhsd")
    cfg = cfg_of("neox", 10000.0, (32, 32), "blocks", "shared", False, positions(2, (1, 4000), g).cuda())
    want = api.attnfuse_qknorm_rope(q, **cfg)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x = q * 1
        got = api.attnfuse_qknorm_rope(x, **cfg)[0]
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("order", ["blocks", "turns"])
@pytest.mark.parametrize("rope", ["neox", "interleaved"])
@pytest.mark.parametrize("D,sections", [(64, (8, 12, 12)), (64, (8, 8, 8, 8)), (128, (16, 24, 24))],
                         ids=lambda x: str(x).replace(" ", ""))
def test_append_every_pair_of_many_tokens(monkeypatch, D, sections, rope, order, dtype):
    """The same where there are workgroups enough for a thread to take several heads: builds of their own."""
    test_append(monkeypatch, 4500, 32, 8, D, 32, dtype, rope, "rows", True, sections, order, "own", "phsd", True)
