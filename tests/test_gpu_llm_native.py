"""The native marshalling of the calls of include/attnfuse_llm.h against the Python one: the same bits, the given outputs
given back, and the same refusals."""
import pytest
import torch

from gpu_util import announce, device_inputs, need_gpu
from paper_2609_13612_amd import api, autograd, blockmask

pytestmark = pytest.mark.gpu
B, H, HKV, S, D = 2, 8, 2, 100, 64


def _inputs():
    _, d = device_inputs(B, H, HKV, S, D, seed=1, with_do=True)
    g = torch.Generator().manual_seed(2)
    d["w"] = (1 + 0.1 * torch.randn(D, generator=g)).bfloat16().cuda()
    d["x"] = torch.randn(B, S, H + 2 * HKV, D, generator=g).bfloat16().cuda()
    d["pages"] = [torch.randn(40, HKV, 16, D, generator=g).bfloat16().cuda() for _ in "kv"]
    d["table"] = torch.randperm(40, generator=g)[:B * 7].to(torch.int32).reshape(B, 7).cuda()
    d["lens"] = torch.tensor([S, 3], dtype=torch.int32).cuda()
    d["pos"] = torch.randint(0, 500, (B, S), generator=g, dtype=torch.int32).cuda()
    d["slots"] = torch.randperm(640, generator=g)[:B * S].cuda()
    return d


def _calls(d):
    """(call(**more), what it gives back) for every entry point in a few variants."""
    q, k, v, do, w, x = (d[n] for n in ("q", "k", "v", "do", "w", "x"))
    sq, sk = x[:, :, :H].transpose(1, 2), x[:, :, H:H + HKV].transpose(1, 2)
    flat = x.reshape(B * S, H + 2 * HKV, D)
    one = q[:, :, 5].contiguous()
    for rope in ("neox", "interleaved", "none"):
        kw = dict(rope=rope, theta=500000.0)
        pos = dict(positions=d["pos"], max_positions=500, **kw)
        yield lambda kw=kw: api.attnfuse_qknorm_rope(sq, sk, w, w, **kw)
        yield lambda pos=pos: api.attnfuse_qknorm_rope(q, None, w.float(), **pos)[:1]
        yield lambda pos=pos: api.attnfuse_qknorm_rope_bwd(sq, sk, do, k, w, None, **pos)
        yield lambda kw=kw: api.attnfuse_qknorm_rope_bwd(q, None, do, None, weight_grads=False, **kw)[:1]

        def append(kw=kw, **more):
            pages = [p.clone() for p in d["pages"]]
            qr = api.attnfuse_qknorm_rope_append(flat[:, :H], flat[:, H:H + HKV], flat[:, H + HKV:], *pages, d["slots"],
                                                 positions=d["pos"].reshape(-1), max_positions=500, **kw, **more)
            return (qr, *pages)

        yield lambda append=append: append(q_weight=w, k_weight=w)
        yield lambda append=append: append(norm=False)
        for more in (dict(mask="causal"), dict(mask="sliding_window", window=20, sinks=3), dict(mask="none", scale=0.2)):
            yield lambda kw=kw, more=more: api.attnfuse_decode_paged(one, *d["pages"], d["table"], d["lens"], **kw, **more)
        win = dict(mask="sliding_window", window=20, sinks=3, **kw)
        yield lambda win=win: api.attnfuse_decode(one, k, v, d["lens"], **win)
        o, lse = api.attnfuse_fwd(q, k, v, **win)
        yield lambda win=win: api.attnfuse_fwd(q, k, v, **win)
        yield lambda win=win, o=o, lse=lse: api.attnfuse_bwd(q, k, v, o, do, lse, **win)


def test_same_bits_as_the_python_marshalling(monkeypatch):
    need_gpu()
    announce("native against python marshalling, llm")
    assert api._native is not None, "the native binding is not built"
    n, real = 0, api._native
    for call in _calls(_inputs()):
        call()                                             # builds the table
        taken = []

        class Spy:
            def __getattr__(self, name):
                def f(*a):
                    taken.append(getattr(real, name)(*a))
                    return taken[-1]
                return f

        monkeypatch.setattr(api, "_native", Spy())
        got = call()
        assert taken and all(t is not None for t in taken), "declined"
        monkeypatch.setattr(api, "_native", None)
        want = call()
        monkeypatch.setattr(api, "_native", real)
        assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, want))
        n += 1
    assert n == 3 * 12


@pytest.mark.parametrize("native", [True, False])
def test_given_outputs_and_refusals(monkeypatch, native):
    need_gpu()
    announce(f"llm outputs and refusals native={native}")
    d = _inputs()
    q, k, v, w = (d[n] for n in ("q", "k", "v", "w"))
    one, kc, vc = q[:, :, 5].contiguous(), *d["pages"]
    tok, tk = one, k[:, :, 5].contiguous()
    if not native:
        monkeypatch.setattr(api, "_native", None)
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    got = api.attnfuse_qknorm_rope(q, k, w, w, out_q=oq, out_k=ok)
    assert got[0] is oq and got[1] is ok
    o, lse = torch.empty_like(one), torch.empty(B, H, device="cuda")
    got = api.attnfuse_decode_paged(one, kc, vc, d["table"], out=o, lse=lse)
    assert got[0] is o and got[1] is lse
    got = api.attnfuse_decode(one, k, v, out=o, lse=lse, mask="sliding_window", window=9, sinks=2)
    assert got[0] is o and got[1] is lse
    slots, pos = torch.zeros(B, dtype=torch.int64, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    slots[1] = 1
    at = dict(positions=pos, max_positions=9)
    assert api.attnfuse_qknorm_rope_append(tok, tk, tk, kc, vc, slots, out_q=o, **at) is o
    bad = [
        (ValueError, lambda: api.attnfuse_qknorm_rope(q.cpu())),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q[..., ::2])),
        (ValueError, lambda: api.attnfuse_qknorm_rope(torch.zeros(1, 1, 2, 132, device="cuda")[..., 2:66])),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q, k.float())),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q, k[:, :, 1:])),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q, k, w, w.float())),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q, k, w[:32], w)),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q, None, w, w)),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q, positions=d["pos"])),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q, positions=d["pos"].long(), max_positions=9)),
        (ValueError, lambda: api.attnfuse_qknorm_rope(q, out_q=q.new_empty(B, S, H, D).transpose(1, 2))),
        (api.AttnFuseError, lambda: api.attnfuse_qknorm_rope(q, eps=-1.0)),
        (api.AttnFuseError, lambda: api.attnfuse_qknorm_rope(q[..., :32].contiguous(), rope="none")),
        (TypeError, lambda: api.attnfuse_qknorm_rope_bwd(q, k, q, None)),
        (ValueError, lambda: api.attnfuse_qknorm_rope_bwd(q, k, q.transpose(1, 2).contiguous().transpose(1, 2), k)),
        (api.AttnFuseError, lambda: api.attnfuse_qknorm_rope_bwd(q, k, q.clone(), k.clone(), workspace=w)),
        (api.AttnFuseError, lambda: api.attnfuse_qknorm_rope_bwd(q, k, q.clone(), k.clone(), dq=q)),
        (ValueError, lambda: api.attnfuse_qknorm_rope_append(tok, tk, tk, kc, vc, slots.int(), **at)),
        (ValueError, lambda: api.attnfuse_qknorm_rope_append(tok, tk, tk, kc, vc, slots)),
        (ValueError, lambda: api.attnfuse_qknorm_rope_append(tok, tk, tk, kc, vc[:39], slots, **at)),
        (ValueError, lambda: api.attnfuse_qknorm_rope_append(tok, tk[:1], tk, kc, vc, slots, **at)),
        (api.AttnFuseError, lambda: api.attnfuse_qknorm_rope_append(tok, tk, tk, kc[:, :, :8], vc[:, :, :8], slots, **at)),
        (api.AttnFuseError, lambda: api.attnfuse_qknorm_rope_append(tok, tk, tk, kc, vc, slots, w, w, norm=False, **at)),
        (api.AttnFuseError, lambda: api.attnfuse_qknorm_rope_append(tok[:0], tk[:0], tk[:0], kc, vc, slots[:0],
                                                                    positions=pos[:0], max_positions=9)),
        (ValueError, lambda: api.attnfuse_decode_paged(one, kc, vc, d["table"].long())),
        (ValueError, lambda: api.attnfuse_decode_paged(one, kc, vc, d["table"][:1])),
        (ValueError, lambda: api.attnfuse_decode_paged(one, kc, vc[..., :32], d["table"])),
        (ValueError, lambda: api.attnfuse_decode_paged(one.float(), kc.float(), vc.float(), d["table"])),
        (ValueError, lambda: api.attnfuse_decode_paged(one, kc, vc, d["table"], sinks=2)),
        (ValueError, lambda: api.attnfuse_decode_paged(one, kc, vc, d["table"], d["lens"].cpu())),
        (api.AttnFuseError, lambda: api.attnfuse_decode_paged(one, kc, vc, d["table"], workspace=w)),
        (api.AttnFuseError, lambda: api.attnfuse_decode_paged(one, kc, vc, d["table"], mask="sliding_window")),
        (api.AttnFuseError, lambda: api.attnfuse_decode_paged(one, kc, vc, d["table"][:, :0].contiguous())),
        (api.AttnFuseError, lambda: api.attnfuse_decode_paged(one[:, :7].contiguous(), kc, vc, d["table"])),
        (ValueError, lambda: api.attnfuse_decode(one.float(), k.float(), v.float(), mask="sliding_window", window=3, sinks=1)),
        (ValueError, lambda: api.attnfuse_decode(one, k, v, mask="causal", sinks=1)),
        (KeyError, lambda: api.attnfuse_decode_paged(one, kc, vc, d["table"], rope="other")),
        (KeyError, lambda: api.attnfuse_qknorm_rope(q, rope="other")),
    ]
    for i, (error, call) in enumerate(bad):
        print(f"refusal {i}", flush=True)
        with pytest.raises(error):
            call()


def _training(d):
    """(leaves, forward, gradients of its outputs) of the differentiable calls."""
    q, k, v, do, w = (d[n] for n in ("q", "k", "v", "do", "w"))
    sq, sk = d["x"][:, :, :H].transpose(1, 2), d["x"][:, :, H:H + HKV].transpose(1, 2)
    far = dict(positions=d["pos"], max_positions=500)
    yield (sq, sk, w, w.clone()), lambda a, b, c, e: autograd.qknorm_rope(a, b, c, e, theta=500000.0), (do, k)
    yield (q, k), lambda a, b: autograd.qknorm_rope(a, b, rope="interleaved", **far), (do, k)
    yield (q, w.float()), lambda a, c: autograd.qknorm_rope(a, None, c, rope="none"), (do,)
    yield (sk, w), lambda a, c: autograd.qknorm_rope(a, None, c), (k.transpose(2, 3).contiguous().transpose(2, 3),)
    for rope in ("neox", "none"):
        kw = dict(rope=rope, mask="sliding_window", window=20, sinks=3)
        yield (q, k, v), lambda a, b, c, kw=kw: autograd.attention(a, b, c, **kw), (do,)
        yield (q, k, v), lambda a, b, c, kw=kw: autograd.attention(a, b, c, scale=0.3, **kw), (do.transpose(1, 2).contiguous()
                                                                                               .transpose(1, 2),)
    f = [x.float() for x in (q, k, v)]
    yield f, lambda a, b, c: autograd.attention(a, b, c, mask="sliding_window", window=7, sinks=1), (do.float(),)


def _grads(leaves, forward, out_grads, wanted=None):
    leaves = [x.detach().requires_grad_(wanted is None or i in wanted) for i, x in enumerate(leaves)]
    out = forward(*leaves)
    out = out if isinstance(out, tuple) else (out,)
    used = [x for x in leaves if x.requires_grad]
    return [o.detach() for o in out] + list(torch.autograd.grad(out, used, out_grads))


def test_differentiable_calls_as_in_python(monkeypatch):
    """The C++ functions against the Python ones: outputs and gradients, all of them or those of one leaf."""
    need_gpu()
    announce("native differentiable calls")
    real, n = api._native, 0
    for case in _training(_inputs()):
        for wanted in (None, {0}, {len(case[0]) - 1}):
            _grads(*case, wanted)                          # builds the table
            got = _grads(*case, wanted)
            monkeypatch.setattr(api, "_native", None)
            want = _grads(*case, wanted)
            monkeypatch.setattr(api, "_native", real)
            assert len(got) == len(want) and all(torch.equal(a, b) and a.stride() == b.stride() for a, b in zip(got, want))
            n += 1
    assert n == 27


def test_differentiable_calls_are_taken_natively(monkeypatch):
    need_gpu()
    announce("native differentiable calls taken")
    for case in _training(_inputs()):
        _grads(*case)
        with monkeypatch.context() as m:
            for name in ("_QkNormRope", "_Attention"):
                m.setattr(autograd, name, None)            # an AttributeError where the Python function would be used
            _grads(*case)


def test_unused_output_and_second_backward():
    """An output without a gradient counts as zeros; a graph kept for a second backward gives the same; LSE takes none."""
    need_gpu()
    announce("native differentiable calls, graphs")
    d = _inputs()
    q, k, w = (d[n].detach().requires_grad_() for n in ("q", "k", "w"))
    qr, kr = autograd.qknorm_rope(q, k, w)
    first = torch.autograd.grad(qr, (q, k, w), d["do"], retain_graph=True)
    want = api.attnfuse_qknorm_rope_bwd(d["q"], d["k"], d["do"], torch.zeros_like(d["k"]), d["w"])
    assert all(torch.equal(a, b) for a, b in zip(first, (want[0], want[1], want[2])))
    assert all(torch.equal(a, b) for a, b in zip(first, torch.autograd.grad(qr, (q, k, w), d["do"])))
    o, lse = autograd.attention(q, k, d["v"], mask="sliding_window", window=9, sinks=2, return_lse=True)
    assert o.requires_grad and not lse.requires_grad
    with torch.no_grad():
        assert not autograd.attention(q, k, d["v"], mask="sliding_window", window=9, sinks=2).requires_grad
    with pytest.raises(RuntimeError):   # a saved tensor changed in place
        o = autograd.attention(q, k, d["v"], mask="sliding_window", window=9, sinks=2)
        with torch.no_grad():
            q.mul_(2)
        torch.autograd.grad(o, q, d["do"])


def test_training_step_replayed_from_a_graph():
    """Norm, rotation, attention with sinks and their backward captured once and replayed on new inputs; an eager graph of
    other leaves lives meanwhile (a captured backward needs leaves of its own: torch ties a leaf's gradient to the stream
    that its first graph was made on)."""
    need_gpu()
    announce("native differentiable calls captured")
    kw = dict(mask="sliding_window", window=30, sinks=4)

    def step(x, w, do):
        leaf, wl = x.detach().requires_grad_(), w.detach().requires_grad_()
        q, k, v = (leaf[:, :, a:b].transpose(1, 2) for a, b in ((0, H), (H, H + HKV), (H + HKV, H + 2 * HKV)))
        qr, kr = autograd.qknorm_rope(q, k, wl, wl, theta=500000.0)
        o = autograd.attention(qr, kr, v.contiguous(), **kw)
        return (o.detach(),) + torch.autograd.grad(o, (leaf, wl), do)

    d = _inputs()
    x, w, do = d["x"].clone(), d["w"], d["do"].clone()
    living = autograd.attention(d["q"].requires_grad_(), d["k"], d["v"], **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, w, do)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step(x, w, do)
    for i in range(3):
        g = torch.Generator("cuda").manual_seed(i)
        x.normal_(generator=g)
        do.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        want = step(x.clone(), w, do.clone())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    torch.autograd.grad(living, d["q"], do)


# ---------------------------------------------------------------- second derivatives
def _twice(d):
    """(leaves, forward) of every differentiable operation, the dense and block-sparse attention among them."""
    q, k, v, w = (d[n] for n in ("q", "k", "v", "w"))
    blocks = blockmask.block_mask_from_dense(torch.ones(2, 2, dtype=torch.bool), S, device="cuda")
    bias = torch.zeros(B, 1, S, S, device="cuda")
    yield (q, k, w, w.clone()), lambda a, b, c, e: autograd.qknorm_rope(a, b, c, e)
    yield (q, w), lambda a, c: autograd.qknorm_rope(a, None, c, positions=d["pos"], max_positions=500)
    yield (q, k, v), lambda a, b, c: autograd.attention(a, b, c, mask="sliding_window", window=20, sinks=3)
    yield (q, k, v), lambda a, b, c: autograd.attention(a, b, c)
    yield (q, k, v), lambda a, b, c: autograd.blocksparse_attention(a, b, c, blocks)
    yield (q, k, v), lambda a, b, c: autograd.attention_bias_norm(a, b, c, bias=bias)


@pytest.mark.parametrize("native", [True, False])
def test_second_derivatives_are_refused(monkeypatch, native):
    """Under create_graph the gradients are those of a plain backward, and a derivative of them is an error, not a loss of
    their part: through backward() and through grad() of one leaf, with a constant gradient and one that itself depends on
    a leaf."""
    need_gpu()
    announce(f"second derivatives native={native}")
    if not native:
        monkeypatch.setattr(api, "_native", None)
    for n, (leaves, forward) in enumerate(_twice(_inputs())):
        print(f"operation {n}", flush=True)
        leaves = [x.detach().requires_grad_() for x in leaves]

        def loss(power):
            out = forward(*leaves)
            return sum((o.float() if power == 1 else o.float().square()).sum() for o in (out if isinstance(out, tuple) else (out,)))

        for power in (1, 2):   # the outputs' gradient: a constant, or the outputs themselves
            want = torch.autograd.grad(loss(power), leaves)
            got = torch.autograd.grad(loss(power), leaves, create_graph=True)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            for i, x in enumerate(got):
                assert x.requires_grad, f"gradient {i} has lost its graph"
                penalised = x.float().square().sum() + sum(y.float().square().sum() for y in leaves)
                with pytest.raises(RuntimeError, match="differentiated twice"):
                    torch.autograd.grad(penalised, leaves[0], retain_graph=True)
                with pytest.raises(RuntimeError, match="differentiated twice"):
                    penalised.backward(retain_graph=True)
        # what does not pass through the gradients is not affected
        (g,) = torch.autograd.grad(sum(y.float().square().sum() for y in leaves), leaves[0], create_graph=True)
        torch.autograd.grad(g.float().sum(), leaves[0])
    assert n == 5


# ---------------------------------------------------------------- positions past max_positions
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("given", [False, True])
def test_positions_from_max_positions_on_give_nan(monkeypatch, native, given):
    """Whatever longer table an earlier call left, or the caller's table holds."""
    need_gpu()
    announce(f"max_positions native={native} given={given}")
    if not native:
        monkeypatch.setattr(api, "_native", None)
    d = _inputs()
    q, k, w = (d[n] for n in ("q", "k", "w"))
    api.attnfuse_qknorm_rope(q, positions=d["pos"], max_positions=5000)   # leaves a table of 5000 rows or more
    kw = dict(positions=d["pos"], max_positions=400, rope_table=api.rope_table(D, 10000.0, 500) if given else None)
    far = (d["pos"] >= 400)
    assert far.any() and not far.all()

    def nan_rows(t, far):
        bad = far[:, None, :, None].expand(t.shape)
        return torch.equal(t.isnan(), bad)

    fine = dict(kw, max_positions=500)
    want = api.attnfuse_qknorm_rope(q, k, w, w, **fine)
    got = api.attnfuse_qknorm_rope(q, k, w, w, **kw)
    for a, b in zip(got, want):
        assert nan_rows(a, far) and torch.equal(a[~a.isnan()], b[~a.isnan()])
    leaves = [x.detach().requires_grad_() for x in (q, k, w, w)]
    out = autograd.qknorm_rope(*leaves, **kw)
    assert all(nan_rows(o, far) for o in out)
    grads = torch.autograd.grad(out, leaves, (d["do"], k))
    assert nan_rows(grads[0], far) and nan_rows(grads[1], far) and grads[2].isnan().all() and grads[3].isnan().all()
    for a, b in zip(api.attnfuse_qknorm_rope_bwd(q, k, d["do"], k, w, w, **kw), grads):
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())
    tok, tk = q.transpose(1, 2).reshape(B * S, H, D), k.transpose(1, 2).reshape(B * S, HKV, D)
    kw["positions"] = d["pos"].reshape(-1)
    kc, vc = (torch.zeros_like(x) for x in d["pages"])
    qr = api.attnfuse_qknorm_rope_append(tok, tk, tk, kc, vc, d["slots"], **kw)
    assert torch.equal(qr.isnan(), far.reshape(-1, 1, 1).expand(qr.shape))
    assert int(kc.isnan().sum()) == int(far.sum()) * HKV * D and not vc.isnan().any()
    for few in (0, -1):
        with pytest.raises(ValueError, match="max_positions"):
            api.attnfuse_qknorm_rope(q, **dict(kw, positions=d["pos"], max_positions=few))
