"""Attention under a sliding window whose first tokens stay visible, forward and backward, against the definition in 64 bits.

Tolerances: the contract's per element (gpu_util: 2e-2 + 2^-8 |ref|, fp32 1e-4, LSE 1e-3) and, over each tensor, a relative
2-norm: the output's rounding, that of P (and of dS, and with RoPE of the rotated operands, 2^-11), each at most half a
step of bf16, 2^-8, in every element: 2 x 2^-8.  In fp32 each value sums up to S products of D-term sums, about sqrt(S + D)
roundings of 2^-24 that do not all fall one way: 64 of them allowed.
"""
import pytest
import torch

import oracle
from gpu_util import announce, assert_bf16_close, assert_fp32_close, assert_lse_close, device_inputs, f64, need_gpu
from llm_ref import U32, rotate, scale_of, visible
from paper_2609_13612_amd import api, autograd

pytestmark = pytest.mark.gpu


def reference(q, k, v, do, rope, theta, window, sinks, scale=None):
    """O, LSE, dQ, dK, dV (fp64), a head at a time."""
    q, k, v, do = (x.double() for x in (q, k, v, do))
    B, H, S, D = q.shape
    G, pos, sc, ok = H // k.shape[1], torch.arange(S), scale_of(D, scale), visible(S, window, sinks)
    o, lse, dq, dk, dv = torch.empty_like(q), q.new_empty(B, H, S), torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b in range(B):
        for h in range(H):
            qr, kr, vv = rotate(q[b, h], pos, rope, theta), rotate(k[b, h // G], pos, rope, theta), v[b, h // G]
            s = (sc * qr @ kr.T).masked_fill(~ok, float("-inf"))
            lse[b, h] = torch.logsumexp(s, 1)
            p = torch.softmax(s, 1)
            o[b, h] = p @ vv
            dp = do[b, h] @ vv.T
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) * sc
            dv[b, h // G] += p.T @ do[b, h]
            dq[b, h] = rotate(ds @ kr, pos, rope, theta, -1.0)
            dk[b, h // G] += rotate(ds.T @ qr, pos, rope, theta, -1.0)
    return o, lse, dq, dk, dv


def check(got, ref, dtype, what):
    got = [f64(x) for x in got]
    for g, r, name in zip(got, ref, ("O", "LSE", "dQ", "dK", "dV")):
        r = r.numpy()
        if name == "LSE":
            assert_lse_close(g, r, what + name)
            continue
        (assert_bf16_close if dtype == "bf16" else assert_fp32_close)(g, r, what + name)
        if not r.any():
            # One visible key: dP and the row term cancel exactly and there is no size to be relative to.  What remains is the
            # difference of two D-term fp32 sums, at most 2 D 2^-24 sum|dO v| scale |k| (D = 64: 8e-6 x 64 x 9 x 0.125 x 3 =
            # 2e-3 for values within 3): the bound per element above holds it.
            continue
        rel = ((g - r) ** 2).sum() ** 0.5 / (r ** 2).sum() ** 0.5
        assert rel <= (2 * 2.0 ** -8 if dtype == "bf16" else 64 * U32), f"{what}{name}: relative 2-norm {rel:.2e}"


CASES = [
    # B, H, Hkv, S, D, dtype, rope, window, sinks
    (1, 8, 2, 1000, 128, "bf16", "neox", 128, 4),
    (2, 4, 4, 777, 64, "bf16", "interleaved", 100, 70),      # sinks over two key tiles, odd length
    (1, 4, 1, 515, 128, "bf16", "none", 33, 1),
    (1, 12, 12, 640, 64, "bf16", "none", 64, 64),            # whole tiles
    (1, 6, 2, 1300, 64, "bf16", "neox", 17, 300),            # sinks over several key blocks of the dK/dV pass
    (1, 2, 2, 257, 128, "bf16", "none", 1, 1),               # a window of the query alone
    (3, 3, 1, 131, 128, "bf16", "neox", 129, 1),             # the last row alone has lost a key, a sink
    (1, 2, 1, 90, 64, "bf16", "none", 40, 49),               # one key is lost, by one row
    (1, 4, 2, 64, 128, "bf16", "neox", 40, 30),              # window + sinks > S: the causal mask
    (2, 2, 2, 1, 64, "bf16", "neox", 1, 1),
    (1, 16, 2, 2100, 128, "bf16", "interleaved", 1024, 16),
    (1, 8, 1, 3000, 64, "bf16", "neox", 256, 4),             # one K/V head: key blocks shared by workgroups
    (2, 4, 4, 3181, 128, "bf16", "none", 102, 5),            # many parts of the sinks' sums, key blocks not shared
    (1, 4, 2, 300, 64, "fp32", "neox", 32, 3),
    (2, 2, 1, 201, 128, "fp32", "none", 50, 40),
    (1, 3, 3, 150, 64, "fp32", "interleaved", 1, 17),
    (1, 2, 2, 33, 128, "fp32", "none", 30, 30),
]


@pytest.mark.parametrize("B,H,Hkv,S,D,dtype,rope,window,sinks", CASES)
def test_forward_and_backward(B, H, Hkv, S, D, dtype, rope, window, sinks):
    need_gpu()
    announce(f"sinks B={B} H={H}/{Hkv} S={S} D={D} {dtype} {rope} W={window} sinks={sinks}")
    cpu, dev = device_inputs(B, H, Hkv, S, D, dtype=dtype, seed=S, with_do=True)
    q, k, v, do = (dev[n] for n in ("q", "k", "v", "do"))
    kw = dict(rope=rope, theta=500000.0, mask="sliding_window", window=window, sinks=sinks)
    o, lse = api.attnfuse_fwd(q, k, v, **kw)
    nbytes = api.attnfuse_bwd_sinks_workspace_bytes(B, H, Hkv, S, D, rope, window, sinks)
    guard = torch.full((nbytes + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    grads = api.attnfuse_bwd(q, k, v, o, do, lse, workspace=guard[:nbytes], **kw)
    torch.cuda.synchronize()
    assert (guard[nbytes:] == 0x5A).all(), "written past the workspace"
    check((o, lse) + grads, reference(cpu["q"], cpu["k"], cpu["v"], cpu["do"], rope, 500000.0, window, sinks), dtype, "")
    again = api.attnfuse_bwd(q, k, v, o, do, lse, workspace=torch.full_like(guard, 0xFF)[:nbytes], **kw)
    assert all(torch.equal(a, b) for a, b in zip(grads, again)), "another workspace's contents, other bits"


def test_the_reference_is_the_oracles_at_its_masks():
    """With every key visible it is the oracle's causal attention."""
    x = {n: torch.randn(1, h, 50, 64, generator=torch.Generator().manual_seed(i)) for i, (n, h) in
         enumerate((("q", 4), ("k", 2), ("v", 2), ("do", 4)))}
    ref = reference(*x.values(), "neox", 10000.0, 30, 20)
    a = [x[n].double().numpy() for n in ("q", "k", "v")]
    O, L = oracle.attention_forward(*a, rope="neox", theta=10000.0, mask="causal")
    grads = oracle.attention_backward(*a, x["do"].double().numpy(), rope="neox", theta=10000.0, mask="causal")
    for r, w in zip(ref, (O, L) + tuple(grads)):
        assert abs(r.numpy() - w).max() < 1e-10


def test_a_window_over_everything_is_the_causal_mask():
    need_gpu()
    announce("sinks causal")
    _, d = device_inputs(2, 8, 2, 600, 128, seed=1, with_do=True)
    args = [d[n] for n in ("q", "k", "v")]
    want = api.attnfuse_fwd(*args)
    for window, sinks in ((600, 1), (1, 599), (10 ** 9, 10 ** 9), (301, 299)):
        kw = dict(mask="sliding_window", window=window, sinks=sinks)
        o, lse = api.attnfuse_fwd(*args, **kw)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        got = api.attnfuse_bwd(*args, o, d["do"], lse, **kw)
        assert all(torch.equal(a, b) for a, b in zip(got, api.attnfuse_bwd(*args, o, d["do"], lse)))


def test_gradient_against_differences():
    """fp32: the derivative of <O, do> along random directions, by central differences of the reference in 64 bits."""
    need_gpu()
    announce("sinks differences")
    cpu, dev = device_inputs(1, 2, 1, 40, 64, dtype="fp32", seed=2, with_do=True)
    kw = dict(rope="neox", theta=10000.0, mask="sliding_window", window=7, sinks=3)
    leaves = [dev[n].requires_grad_() for n in ("q", "k", "v")]
    grads = torch.autograd.grad(autograd.attention(*leaves, **kw), leaves, dev["do"])
    g, x = torch.Generator().manual_seed(3), [cpu[n].double() for n in ("q", "k", "v")]
    for i in range(3):
        for _ in range(4):
            d = torch.randn(x[i].shape, generator=g, dtype=torch.float64)
            d /= d.norm()
            loss = [(reference(*[y + s * 1e-4 * d if j == i else y for j, y in enumerate(x)], cpu["do"], "neox", 10000.0, 7, 3)[0]
                     * cpu["do"].double()).sum() for s in (1, -1)]
            want = (loss[0] - loss[1]) / 2e-4
            # differences: 1e-8 of a third derivative of order 10; fp32: 64 u of the gradient's norm
            assert abs((f64_(grads[i]) * d).sum() - want) < 1e-6 + 64 * U32 * f64_(grads[i]).norm()


def f64_(t):
    return t.detach().cpu().double()


def test_less_workspace_and_autograd():
    """Without room for the shared key blocks' partials, and through autograd: the same gradients."""
    need_gpu()
    announce("sinks workspace")
    B, H, Hkv, S, D, window, sinks = 1, 8, 1, 1500, 128, 200, 5
    cpu, dev = device_inputs(B, H, Hkv, S, D, seed=4, with_do=True)
    q, k, v, do = (dev[n] for n in ("q", "k", "v", "do"))
    kw = dict(rope="neox", mask="sliding_window", window=window, sinks=sinks)
    ref = reference(cpu["q"], cpu["k"], cpu["v"], cpu["do"], "neox", 10000.0, window, sinks)
    o, lse = api.attnfuse_fwd(q, k, v, **kw)
    base = api.attnfuse_bwd_workspace_bytes(B, H, Hkv, S, D, "neox")
    far = api.attnfuse_bwd_sinks_workspace_bytes(B, H, Hkv, S, D, "neox", window, sinks) - base
    rows = B * (2 * H + Hkv) * S * D * 2 + 2 * B * H * S * 4
    least = far + rows + 256 * 7 + 4 * B * Hkv * (H * S * D // 16384 + 64)   # each part, rounded up
    assert least < far + base
    check((o, lse) + api.attnfuse_bwd(q, k, v, o, do, lse, workspace=torch.empty(least, dtype=torch.uint8, device="cuda"), **kw),
          ref, "bf16", "least ")
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    got = torch.autograd.grad(autograd.attention(*leaves, **kw), leaves, do)
    assert all(torch.equal(a, b) for a, b in zip(got, api.attnfuse_bwd(q, k, v, o, do, lse, **kw)))


def test_replayed_from_a_graph():
    need_gpu()
    announce("sinks graph")
    B, H, Hkv, S, D = 1, 8, 2, 900, 128
    kw = dict(rope="neox", theta=500000.0, mask="sliding_window", window=128, sinks=4)
    _, d0 = device_inputs(B, H, Hkv, S, D, seed=70, with_do=True)
    q, k, v, do = (d0[n].clone() for n in ("q", "k", "v", "do"))
    o, lse = api.attnfuse_fwd(q, k, v, **kw)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        o, lse = api.attnfuse_fwd(q, k, v, **kw)
        grads = api.attnfuse_bwd(q, k, v, o, do, lse, **kw)
    for seed in (71, 72, 73):
        _, d = device_inputs(B, H, Hkv, S, D, seed=seed, with_do=True)
        want = api.attnfuse_fwd(d["q"], d["k"], d["v"], **kw)
        want += api.attnfuse_bwd(d["q"], d["k"], d["v"], want[0], d["do"], want[1], **kw)
        torch.cuda.synchronize()
        for dst, name in ((q, "q"), (k, "k"), (v, "v"), (do, "do")):
            dst.copy_(d[name])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((o, lse) + grads, want)), seed


def test_normed_and_rotated_in_training():
    """norm + rotation, then attention under the mask, as a layer trains: O and every gradient against the chain in 64 bits."""
    need_gpu()
    announce("qknorm then sinks")
    from llm_ref import qknorm, qknorm_bwd
    B, H, Hkv, S, D, window, sinks = 1, 4, 2, 300, 64, 64, 4
    g = torch.Generator().manual_seed(9)
    x = torch.randn(B, S, H + 2 * Hkv, D, generator=g)
    qw, kw_ = (1 + 0.2 * torch.randn(D, generator=g) for _ in "qk")
    do = torch.randn(B, H, S, D, generator=g)
    leaf = x.cuda().requires_grad_()
    ws = [w.cuda().requires_grad_() for w in (qw, kw_)]
    q, k, v = (leaf[:, :, a:b].transpose(1, 2) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    qr, kr = autograd.qknorm_rope(q, k, *ws, theta=10000.0)
    o = autograd.attention(qr, kr, v.contiguous(), mask="sliding_window", window=window, sinks=sinks)
    got = torch.autograd.grad(o, [leaf] + ws, do.cuda())
    pos = torch.arange(S)
    q, k, v = (x[:, :, a:b].transpose(1, 2) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    q64, k64 = qknorm(q, qw, pos, "neox", 10000.0, 1e-6)[0], qknorm(k, kw_, pos, "neox", 10000.0, 1e-6)[0]
    ref = reference(q64, k64, v, do, "none", 1.0, window, sinks)
    dq, dqw = qknorm_bwd(q, qw, ref[2], pos, "neox", 10000.0, 1e-6)[:2]
    dk, dkw = qknorm_bwd(k, kw_, ref[3], pos, "neox", 10000.0, 1e-6)[:2]
    want = [torch.cat((dq, dk, ref[4]), 1).transpose(1, 2), dqw, dkw]
    for a, b, what in zip([o] + list(got), [ref[0]] + want, ("O", "dx", "dq_weight", "dk_weight")):
        assert (f64_(a) - b).norm() <= 64 * U32 * b.norm(), what


def test_refusals():
    need_gpu()
    announce("sinks refusals")
    _, d = device_inputs(1, 4, 2, 64, 64, seed=1, with_do=True)
    args = [d[n] for n in ("q", "k", "v")]
    slopes = torch.ones(4, device="cuda")
    for bad in (dict(sinks=2), dict(sinks=2, mask="causal", window=4), dict(sinks=-1, mask="sliding_window", window=4),
                dict(sinks=2, mask="sliding_window"), dict(sinks=2, mask="sliding_window", window=0),
                dict(sinks=2, mask="sliding_window", window=4, alibi_slopes=slopes)):
        with pytest.raises(ValueError):
            api.attnfuse_fwd(*args, **bad)
        with pytest.raises(ValueError):
            api.attnfuse_bwd(*args, args[0], d["do"], torch.zeros(1, 4, 64, device="cuda"), **bad)
    with pytest.raises(ValueError):
        api.attnfuse_fwd(args[0], args[1].float(), args[2], mask="sliding_window", window=4, sinks=1)


@pytest.mark.parametrize("native", [True, False])
def test_windows_and_sinks_past_32_bits(monkeypatch, native):
    """As every key's: forward, backward, autograd and both decodes; a plain window too."""
    need_gpu()
    announce(f"sinks past 32 bits native={native}")
    if not native:
        monkeypatch.setattr(api, "_native", None)
    _, d = device_inputs(1, 4, 2, 100, 64, seed=5, with_do=True)
    q, k, v, do = (d[n] for n in ("q", "k", "v", "do"))
    one = q[:, :, 7].contiguous()
    pages = [x.transpose(1, 2).reshape(1, 100, 2, 64)[:, :96].reshape(6, 16, 2, 64).transpose(1, 2) for x in (k, v)]
    table = torch.arange(6, dtype=torch.int32, device="cuda")[None]
    want = api.attnfuse_fwd(q, k, v)
    grads = api.attnfuse_bwd(q, k, v, *want[:1], do, want[1])
    for window, sinks in ((2 ** 32 + 5, 4), (5, 2 ** 32 + 1), (2 ** 31, 2 ** 31), (2 ** 32 + 5, 0)):
        kw = dict(mask="sliding_window", window=window, sinks=sinks)
        o, lse = api.attnfuse_fwd(q, k, v, **kw)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        assert all(torch.equal(a, b) for a, b in zip(api.attnfuse_bwd(q, k, v, o, do, lse, **kw), grads))
        leaves = [x.detach().requires_grad_() for x in (q, k, v)]
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(autograd.attention(*leaves, **kw), leaves, do), grads))
        most = dict(mask="sliding_window", window=100, sinks=min(sinks, 1))
        for call in (lambda **m: api.attnfuse_decode(one, k, v, **m), lambda **m: api.attnfuse_decode_paged(one, *pages, table, **m)):
            assert all(torch.equal(a, b) for a, b in zip(call(**kw), call(**most)))
