"""The native marshalling of the calls of include/attnfuse_llm.h against the Python one: the same bits, the given outputs
given back, and the same refusals."""
import pytest
import torch

from gpu_util import announce, device_inputs, need_gpu
from paper_2609_13612_amd import api

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
