"""Norm and rotation of query and key rows, its backward, and the form that writes new tokens' keys and values to a paged
cache, against the definition in 64 bits.

Tolerances.  An output is rounded once to its type: half a step of the exact value.  Before that come fp32 roundings
(u = 2^-24): the sum of D squares (16 fused steps and three adds: at most 20 u of it, 10 u of its root), the root and the
division (2 u), the products with w and r (3 u), a rotation's two products with rounded cos and sin and their sum (3 u of
each term, of which there are two no larger than the row's largest |w x r|): under 40 u of that, 64 u allowed.  The
gradient's row sum adds the same again: 128 u of r (max|g| + max|xh| mean|g xh|).  A weight's gradient sums its terms
(themselves 20 u off) over at most n rows per thread and then 32 threads, 32 lanes of workgroups and 32 of those: (n + 128) u
of the sum of their magnitudes.
"""
import pytest
import torch

from gpu_util import announce, need_gpu
from llm_ref import U32, assert_within, f64, half_step, qknorm, qknorm_bwd, rotate
from paper_2609_13612_amd import api, autograd

pytestmark = pytest.mark.gpu
EPS = 1e-6


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


CASES = [
    # B, H, Hkv, S, D, dtype, rope, layout, weights, positions
    (1, 32, 8, 300, 128, torch.bfloat16, "neox", "slice", "rows", False),
    (2, 12, 12, 77, 64, torch.bfloat16, "interleaved", "bshd", "fp32", False),
    (3, 5, 2, 33, 128, torch.float32, "neox", "bhsd", "fp32", True),
    (1, 1, 1, 1, 64, torch.bfloat16, "neox", "bhsd", "rows", True),
    (2, 7, 3, 1, 128, torch.float32, "interleaved", "slice", "none", True),
    (1, 3, 1, 2049, 64, torch.float32, "none", "bshd", "fp32", False),
    (2, 6, 0, 40, 128, torch.bfloat16, "interleaved", "slice", "rows", False),   # no keys
    (4, 16, 4, 1000, 128, torch.bfloat16, "none", "bhsd", "rows", False),
    (1, 64, 8, 700, 64, torch.bfloat16, "neox", "slice", "rows", True),          # more units than workgroups
    # short sequences, several a workgroup: as many as fit, with rows to spare, and a last workgroup that is not full
    (67, 5, 2, 1, 128, torch.bfloat16, "neox", "slice", "fp32", True),
    (23, 6, 3, 3, 64, torch.bfloat16, "interleaved", "bhsd", "rows", False),
    (5, 4, 4, 16, 128, torch.float32, "neox", "bshd", "rows", True),
    # several heads a thread, not all of them there for the last
    (2, 9, 3, 2000, 128, torch.float32, "neox", "slice", "fp32", False),
    (12, 7, 3, 900, 64, torch.bfloat16, "interleaved", "bshd", "rows", True),
]


@pytest.mark.parametrize("B,H,Hkv,S,D,dtype,rope,layout,wkind,given", CASES, ids=lambda x: str(x).replace("torch.", ""))
def test_forward_and_backward(B, H, Hkv, S, D, dtype, rope, layout, wkind, given):
    need_gpu()
    announce(f"qknorm B={B} H={H}/{Hkv} S={S} D={D} {dtype} {rope} {layout} {wkind} {given}")
    g = torch.Generator().manual_seed(S + D)
    q, k = rows((B, H, S, D), dtype, g, layout), rows((B, Hkv, S, D), dtype, g, layout) if Hkv else None
    qw, kw = weights(D, wkind, dtype, g)
    kw = kw if Hkv else None
    do = [rows((B, h, S, D), dtype, g, "bhsd") for h in (H, Hkv) if h]
    pos = torch.randint(0, 5000, (B, S), generator=g, dtype=torch.int32).cuda() if given else None
    cfg = dict(eps=EPS, rope=rope, theta=500000.0, positions=pos, max_positions=5000 if given else None)
    at = pos.cpu()[:, None] if given else torch.arange(S)
    out = api.attnfuse_qknorm_rope(q, k, qw, kw, **cfg)
    grads = api.attnfuse_qknorm_rope_bwd(q, k, do[0], do[1] if Hkv else None, qw, kw, **cfg)
    assert (out[1] is None and grads[1] is None and grads[3] is None) == (not Hkv)
    for i, (x, w) in enumerate(((q, qw), (k, kw))[: len(do)]):
        want, size = qknorm(x, w, at, rope, 500000.0, EPS)
        assert out[i].is_contiguous() and out[i].dtype == dtype
        assert_within(out[i], want, half_step(dtype) * want.abs() + 64 * U32 * size, "qk"[i] + "'")
        dx, dw, dsize, wsize = qknorm_bwd(x, w, do[i], at, rope, 500000.0, EPS)
        assert_within(grads[i], dx, half_step(dtype) * dx.abs() + 128 * U32 * dsize, "d" + "qk"[i])
        wt = torch.float32 if wkind in ("fp32", "none") else dtype
        assert grads[2 + i].dtype == wt
        n = B * x.shape[1] * S   # rows of a thread: all, divided over 32 threads of up to 1024 workgroups
        assert_within(grads[2 + i], dw, half_step(wt) * dw.abs() + (n / 32 + 148) * U32 * wsize, "dw of " + "qk"[i])
    again = api.attnfuse_qknorm_rope_bwd(q, k, do[0], do[1] if Hkv else None, qw, kw, **cfg)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(again, grads)), "another call, other bits"


def test_against_differences():
    """The gradients of a random projection of the outputs against central differences of the definition in 64 bits."""
    need_gpu()
    announce("qknorm differences")
    g = torch.Generator().manual_seed(5)
    q = torch.randn(1, 2, 3, 64, generator=g)
    w = 1 + 0.2 * torch.randn(64, generator=g)
    do = torch.randn(1, 2, 3, 64, generator=g)
    dq, _, dw, _ = api.attnfuse_qknorm_rope_bwd(q.cuda(), None, do.cuda(), None, w.cuda(), eps=EPS)

    def loss(x, w):
        return (qknorm(x, w, torch.arange(3), "neox", 10000.0, EPS)[0] * do.double()).sum()

    h = 1e-5
    for _ in range(40):
        i = int(torch.randint(q.numel(), (1,), generator=g))
        e = torch.zeros(q.numel(), dtype=torch.float64)
        e[i] = h
        diff = (loss(q.double() + e.view(q.shape), w) - loss(q.double() - e.view(q.shape), w)) / (2 * h)
        assert abs(float(dq.flatten()[i]) - diff) < 2e-5   # fp32: 128 u of about 8; differences: h^2 and 2^-53 / h
        j = i % 64
        e = torch.zeros(64, dtype=torch.float64)
        e[j] = h
        diff = (loss(q, w.double() + e) - loss(q, w.double() - e)) / (2 * h)
        assert abs(float(dw[j]) - diff) < 2e-5


def test_autograd_gives_the_same_gradients():
    need_gpu()
    announce("qknorm autograd")
    g = torch.Generator().manual_seed(6)
    q, k = (rows((2, h, 50, 128), torch.bfloat16, g, "slice").detach().requires_grad_() for h in (8, 2))
    qw, kw = (w.requires_grad_() for w in weights(128, "rows", torch.bfloat16, g))
    dq, dk = (rows((2, h, 50, 128), torch.bfloat16, g, "bshd") for h in (8, 2))
    qr, kr = autograd.qknorm_rope(q, k, qw, kw)
    got = torch.autograd.grad((qr, kr), (q, k, qw, kw), (dq, dk))
    want = api.attnfuse_qknorm_rope_bwd(q, k, dq.contiguous(), dk.contiguous(), qw, kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert got[0].stride() == (50 * 8 * 128, 128, 8 * 128, 1)   # as q lies, without its gaps
    x = q.detach().contiguous().requires_grad_()
    (only,) = torch.autograd.grad(autograd.qknorm_rope(x, rope="none").float().square().sum(), (x,))
    assert torch.isfinite(only).all()


def test_in_place_and_zero_rows():
    """q' over q; a row of zeros is zeros (eps keeps it finite), and its gradient that of x / sqrt(eps)."""
    need_gpu()
    announce("qknorm in place")
    g = torch.Generator().manual_seed(7)
    q, k = (rows((1, h, 20, 64), torch.bfloat16, g, "bhsd") for h in (5, 2))
    q[0, 1, 3] = 0
    want = api.attnfuse_qknorm_rope(q, k)
    assert not want[0][0, 1, 3].any()
    x = q.clone()
    api.attnfuse_qknorm_rope(x, k, out_q=x)
    assert torch.equal(x, want[0])
    do = rows((1, 5, 20, 64), torch.bfloat16, g, "bhsd")
    dq = api.attnfuse_qknorm_rope_bwd(q, None, do, None, rope="none", weight_grads=False, eps=1e-4)
    assert dq[2] is None
    assert_within(dq[0][0, 1, 3], 100 * f64(do[0, 1, 3]), 1.01 * half_step(torch.bfloat16) * 100 * f64(do[0, 1, 3]).abs(), "dx")


def test_positions_outside_the_table_give_nan():
    need_gpu()
    announce("qknorm bad positions")
    q = torch.randn(2, 3, 5, 64, device="cuda")
    pos = torch.tensor([[0, 1, 2, 3, 4], [-1, 7, 8, 2 ** 31 - 1, 1]], dtype=torch.int32, device="cuda")
    table = api.rope_table(64, 10000.0, 8)
    out, _ = api.attnfuse_qknorm_rope(q, positions=pos, rope_table=table)
    bad = torch.tensor([[False] * 5, [True, False, True, True, False]], device="cuda")
    assert torch.equal(out.isnan().all(-1).all(1), bad) and torch.equal(out.isnan().any(-1).any(1), bad)


# ---------------------------------------------------------------- new tokens into pages
APPENDS = [
    # T, H, Hkv, D, pages, page size, dtype, rope, norm, places first
    (1, 32, 8, 128, 9, 16, torch.bfloat16, "neox", True, False),
    (300, 5, 2, 64, 40, 16, torch.bfloat16, "interleaved", True, True),
    (77, 12, 12, 64, 3, 128, torch.float32, "neox", False, False),
    (1000, 64, 8, 128, 70, 32, torch.bfloat16, "none", True, True),
    (33, 1, 1, 128, 5, 64, torch.float32, "none", False, False),
    (2000, 11, 5, 128, 130, 16, torch.float32, "neox", True, True),
    (3000, 13, 3, 64, 50, 64, torch.bfloat16, "neox", True, False),
    (3000, 25, 7, 64, 50, 64, torch.bfloat16, "interleaved", False, True),
]


@pytest.mark.parametrize("T,H,Hkv,D,pages,page,dtype,rope,norm,nhd", APPENDS, ids=lambda x: str(x).replace("torch.", ""))
def test_append(T, H, Hkv, D, pages, page, dtype, rope, norm, nhd):
    need_gpu()
    announce(f"append T={T} H={H}/{Hkv} D={D} {pages}x{page} {dtype} {rope} norm={norm} {nhd}")
    g = torch.Generator().manual_seed(T)
    wide = torch.randn(T, H + 2 * Hkv, D, generator=g).to(dtype).cuda()
    q, k, v = wide[:, :H], wide[:, H:H + Hkv], wide[:, H + Hkv:]
    shape = (pages, page, Hkv, D) if nhd else (pages, Hkv, page, D)
    kc, vc = (torch.randn(shape, generator=g).to(dtype).cuda() for _ in "kv")
    if nhd:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    k0, v0 = kc.clone(), vc.clone()
    slots = torch.randperm(pages * page, generator=g)[:T]
    if T > 20:   # padding, and slots behind the last page: nothing is written
        slots[3], slots[7], slots[11], slots[12] = -1, pages * page, 2 ** 40, -2 ** 62
    qw, kw = weights(D, "rows", dtype, g) if norm else (None, None)
    pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32) if rope != "none" else None
    cfg = dict(norm=norm, eps=EPS, rope=rope, theta=500000.0, max_positions=100000,
               positions=None if pos is None else pos.cuda())
    qr = api.attnfuse_qknorm_rope_append(q, k, v, kc, vc, slots.cuda(), qw, kw, **cfg)

    def want(x, w):
        if norm:
            return qknorm(x, w, pos[:, None] if pos is not None else torch.zeros(T, 1), rope, 500000.0, EPS)
        y = f64(x)
        return (rotate(y, pos[:, None], rope, 500000.0) if pos is not None else y), y.abs().amax(-1, keepdim=True)

    def close(got, x, w, rows_, what):
        ref, size = want(x, w)
        assert_within(got, ref[rows_], half_step(dtype) * ref[rows_].abs() + 64 * U32 * size[rows_], what)

    close(qr, q, qw, slice(None), "q'")
    kept = ((slots >= 0) & (slots < pages * page)).nonzero()[:, 0]
    at = slots[kept]
    close(kc.transpose(1, 2)[at // page, at % page], k, kw, kept, "cached keys")
    assert torch.equal(vc.transpose(1, 2)[at // page, at % page], v[kept.cuda()])
    k0.transpose(1, 2)[at // page, at % page] = kc.transpose(1, 2)[at // page, at % page]
    v0.transpose(1, 2)[at // page, at % page] = vc.transpose(1, 2)[at // page, at % page]
    assert torch.equal(kc, k0) and torch.equal(vc, v0), "another slot was written"


def test_replayed_from_a_graph():
    """Forward, backward and append captured once, replayed on new inputs with eager work between, bit for bit."""
    need_gpu()
    announce("qknorm graph")
    B, H, Hkv, S, D = 2, 8, 2, 70, 128
    g = torch.Generator().manual_seed(8)

    def inputs():
        x = torch.randn(B, S, H + 2 * Hkv, D, generator=g).bfloat16().cuda()
        return x, torch.randn(B, H, S, D, generator=g).bfloat16().cuda(), torch.randn(B, Hkv, S, D, generator=g).bfloat16().cuda()

    qw, kw = weights(D, "rows", torch.bfloat16, g)
    slots = torch.randperm(1024, generator=g)[: B * S].cuda()
    pos = torch.randint(0, 4000, (B * S,), generator=g, dtype=torch.int32).cuda()
    pages = [torch.zeros(64, Hkv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in "kvkv"]

    def step(x, dq, dk, kc, vc):
        q, k = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hkv].transpose(1, 2)
        flat = x.reshape(B * S, H + 2 * Hkv, D)
        return (api.attnfuse_qknorm_rope(q, k, qw, kw) + api.attnfuse_qknorm_rope_bwd(q, k, dq, dk, qw, kw)
                + (api.attnfuse_qknorm_rope_append(flat[:, :H], flat[:, H:H + Hkv], flat[:, H + Hkv:], kc, vc, slots, qw, kw,
                                                   positions=pos, max_positions=4000),))

    static = inputs()
    step(*static, *pages[:2])   # builds the table
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step(*static, *pages[:2])
    for _ in range(3):
        new = inputs()
        for a, b in zip(static, new):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want = step(*new, *pages[2:])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(pages[0], pages[2]) and torch.equal(pages[1], pages[3])


def test_on_two_streams():
    need_gpu()
    announce("qknorm streams")
    g = torch.Generator().manual_seed(9)
    xs = [rows((1, 16, 2000, 128), torch.bfloat16, g, "bshd") for _ in range(2)]
    dos = [rows((1, 16, 2000, 128), torch.bfloat16, g, "bhsd") for _ in range(2)]
    w = weights(128, "rows", torch.bfloat16, g)[0]
    want = [api.attnfuse_qknorm_rope_bwd(x, None, d, None, w) for x, d in zip(xs, dos)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = api.attnfuse_qknorm_rope_bwd(xs[i], None, dos[i], None, w)
        torch.cuda.synchronize()
        assert all(torch.equal(got[i][j], want[i][j]) for i in range(2) for j in (0, 2))


# ---------------------------------------------------------------- the weights' gradients, row by row
DW = [
    # H, S, B, D, dtype, rope
    (64, 700, 1, 64, torch.bfloat16, "neox"),            # more units than workgroups
    (9, 2000, 2, 128, torch.float32, "neox"),            # as above, a last head group that is not full
    (5, 1, 67, 128, torch.bfloat16, "none"),             # several sequences a workgroup, a last one that is not full
    (7, 3, 23, 64, torch.float32, "interleaved"),
    (1, 1, 1, 64, torch.bfloat16, "none"),
]


def _dw_setup(H, S, B, D, dtype):
    g = torch.Generator().manual_seed(S + H)
    return g, rows((B, H, S, D), dtype, g, "slice"), rows((B, H, S, D), dtype, g, "bhsd"), weights(D, "fp32", dtype, g)[0]


@pytest.mark.parametrize("H,S,B,D,dtype,rope", DW, ids=lambda x: str(x).replace("torch.", ""))
def test_every_row_counts_once(H, S, B, D, dtype, rope):
    """An incoming gradient in one row: dw is that row's dy xh alone, each element to 64 u, at the edges of what threads,
    workgroups and their shares take.  (A row lost, or added twice, is off by all of it.)"""
    need_gpu()
    announce(f"dw rows H={H} S={S} B={B} D={D} {dtype} {rope}")
    g, q, do, w = _dw_setup(H, S, B, D, dtype)
    R = 4096 // D
    at = {(b, h, n) for b in (0, B // 2, B - 1) for h in (0, 1, H - 2, H - 1)
          for n in (0, 1, R - 1, R, R * (S // R) - 1, R * (S // R), S - 1) if 0 <= h < H and 0 <= n < S}
    at |= {tuple(int(torch.randint(x, (1,), generator=g)) for x in (B, H, S)) for _ in range(20)}
    one = torch.zeros_like(do)
    for b, h, n in sorted(at):
        one[b, h, n] = do[b, h, n]
        got = api.attnfuse_qknorm_rope_bwd(q, None, one, None, w, eps=EPS, rope=rope)[2]
        one[b, h, n] = 0
        pos = torch.tensor([n])
        _, want, _, size = qknorm_bwd(q[b, h, n:n + 1], w, do[b, h, n:n + 1], pos, rope, 10000.0, EPS)
        # rotated terms: each element of dy is a sum of two, no larger together than the row's largest |dout|
        size = size + want.new_tensor(float(do[b, h, n].abs().max())) * (f64(q[b, h, n]).abs() /
                                                                        f64(q[b, h, n]).square().mean().sqrt())
        assert_within(got, want, 64 * U32 * size, f"dw of row {b, h, n}")


@pytest.mark.parametrize("H,S,B,D,dtype,rope", DW, ids=lambda x: str(x).replace("torch.", ""))
def test_weight_gradient_to_the_length_of_its_sums(H, S, B, D, dtype, rope):
    """All rows: an element's additions are a thread's rows (two heads for each of its units), the rows of a workgroup, a
    32nd of the workgroups and 32 sums of those, each of 2^-24 of the magnitudes at most; a term itself is 64 of them off."""
    need_gpu()
    announce(f"dw sums H={H} S={S} B={B} D={D} {dtype} {rope}")
    _, q, do, w = _dw_setup(H, S, B, D, dtype)
    R = 4096 // D
    wgs = api.attnfuse_qknorm_rope_bwd_workspace_bytes(B, H, 0, S, D, dtype) // (4 * D)
    per = R // S if 2 * S <= R else 1
    units = -(-B // per) * -(-H // 2) * -(-S // R)
    depth = 2 * -(-units // wgs) + R + -(-wgs // 32) + 32
    got = api.attnfuse_qknorm_rope_bwd(q, None, do, None, w, eps=EPS, rope=rope)[2]
    _, want, _, size = qknorm_bwd(q, w, do, torch.arange(S), rope, 10000.0, EPS)
    if rope != "none":   # (as above, over all rows)
        x = f64(q)
        size = size + (f64(do).abs().amax(-1, keepdim=True) * x.abs() / x.square().mean(-1, keepdim=True).sqrt()).sum((0, 1, 2))
    assert_within(got, want, (depth + 64) * U32 * size, "dw")
