"""The calls that the language-model operators are measured on, over the ranges their users meet.

Kinds of call, each through a public entry point:

  qknorm   autograd.qknorm_rope, forward and backward: the per-head RMS norm of a layer's queries and keys and their
           rotation, as it is trained; q and k are views of the fused projection's output [B, S, (H + 2 H_kv) D]
  append   api.attnfuse_qknorm_rope_append: the same for new tokens, keys and values written to a paged cache
  sinks    autograd.attention under a sliding window whose first tokens stay visible, forward and backward
  prompt   api.attnfuse_fwd under the same mask, of queries and keys already rotated: O and LSE of a prompt
  paged    api.attnfuse_decode_paged: one new token per sequence against a paged cache, split and joined
  stream   api.attnfuse_decode with sinks: one new token per sequence against a contiguous cache

Each has its plain form here, in elementary torch operations.  Tensors are N(0, 1), as in the framework's parity
workloads, and norm weights 1 + N(0, 0.1); the sizes are those workloads' and head geometries, or odd sizes between.
"""
import math

import torch

own = False

HEADS = ((32, 8, 128), (64, 8, 128), (16, 16, 128), (12, 12, 64), (16, 16, 64), (8, 2, 64), (24, 8, 128), (12, 4, 128))
EPS = 1e-6


def _case(kind, **kw):
    c = dict(kind=kind, B=1, H=32, Hkv=8, S=8192, D=128, rope="neox", theta=10000.0, dtype="bf16")
    c.update(kw)
    return c


def listed():
    return [
        # Queries and keys of a Llama-3-8B layer in training, the headline step's sizes.
        _case("qknorm", name="qknorm_train_8k", theta=500000.0),
        # GPT-2-small heads, odd length, interleaved pairs.
        _case("qknorm", name="qknorm_train_d64_odd", B=4, H=12, Hkv=12, S=1777, D=64, rope="interleaved"),
        # The fp32 arithmetic that a port is checked with.
        _case("qknorm", name="qknorm_train_fp32", B=2, H=8, Hkv=2, S=777, dtype="fp32"),
        # One sequence's newest token: the smallest call that a server makes per layer, where latency is all.
        _case("append", name="append_one_token", S=1, pages=512, page=16, theta=500000.0),
        # A step's mixed batch: chunks of prompts and single tokens, some rows padding, into pages of 64.
        _case("append", name="append_prompt_chunks", S=4500, H=64, pages=1200, page=64),
        # A Llama-3-8B layer in training under a window of 1024 with four sinks.
        _case("sinks", name="sinks_train_8k", W=1024, sinks=4, theta=500000.0),
        # Small heads, already rotated, odd length, more sinks than a tile has keys.
        _case("sinks", name="sinks_train_d64", B=4, H=12, Hkv=12, S=2001, D=64, W=256, sinks=70, rope="none"),
        # A long prompt under a window: the work is in the band.
        _case("prompt", name="sinks_prompt_16k", S=16384, W=4096, sinks=4, rope="none"),
        # Serving, one sequence, Llama-3-8B with a 4k cache in pages of 16.
        _case("paged", name="paged_one_4k", S=4096, page=16, ragged=False, W=0, sinks=0, theta=500000.0),
        # Serving, a batch of conversations of different lengths.
        _case("paged", name="paged_batch_8k", B=32, S=8192, page=64, ragged=True, W=0, sinks=0, theta=500000.0),
        # Serving, long conversations, Llama-3-70B heads: the largest cache.
        _case("paged", name="paged_long_32k", B=8, H=64, S=32768, page=32, ragged=True, W=0, sinks=0, theta=500000.0),
        # Streaming: long contiguous caches of which a window and the sinks are read.
        _case("stream", name="stream_window", B=8, S=20000, ragged=True, W=4096, sinks=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("qknorm", "append", "sinks", "sinks", "prompt", "paged", "paged", "stream"))
    H, Hkv, D = rng.choice(HEADS)
    v = dict(H=H, Hkv=Hkv, D=D, theta=rng.choice((10000.0, 500000.0)))
    rope = rng.choice(("neox", "neox", "interleaved", "none"))
    if kind == "qknorm":
        S = _log(rng, 5, 8192)
        return _case(kind, B=max(1, min(rng.randint(1, 6), 8192 // S)), S=S, rope=rope,
                     dtype=rng.choice(("bf16", "bf16", "fp32")), **v)
    if kind == "append":
        page = rng.choice((16, 32, 64, 128, 256))
        T = _log(rng, 1, 4500)
        return _case(kind, S=T, page=page, pages=2 + 2 * T // page + rng.randint(0, 64), rope=rope,
                     dtype=rng.choice(("bf16", "bf16", "bf16", "fp32")), **v)
    if kind in ("sinks", "prompt"):
        S = _log(rng, 40, 8192 if kind == "sinks" else 16384)
        fp32 = kind == "sinks" and S < 500 and rng.random() < 0.4
        return _case(kind, B=max(1, min(rng.randint(1, 4), 8192 // S)), S=S, W=_log(rng, 16, max(17, min(S, 4096))),
                     sinks=rng.choice((1, 4, 4, 16, 64, 130)), rope="none" if kind == "prompt" else rope,
                     dtype="fp32" if fp32 else "bf16", **v)
    S = _log(rng, 20, 32768)
    B = max(1, min(_log(rng, 1, 48), 5 * 32768 // S))
    W = _log(rng, 16, 8192) if kind == "stream" or rng.random() < 0.4 else 0
    sinks = rng.choice((1, 4, 16, 100)) if W and (kind == "stream" or rng.random() < 0.7) else 0
    return _case(kind, B=B, S=S, page=rng.choice((16, 16, 32, 64, 128, 256)), ragged=rng.random() < 0.6, W=W, sinks=sinks,
                 rope=rope, **v)


# ---------------------------------------------------------------- inputs
def _tensors(case, seed):
    """The tensors of a case, on the GPU, from the seed alone."""
    g = torch.Generator("cuda").manual_seed(seed)
    B, H, Hkv, S, D, kind = (case[k] for k in ("B", "H", "Hkv", "S", "D", "kind"))
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16

    def rnd(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    def whole(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)

    if kind == "qknorm":
        x = rnd(B, S, H + 2 * Hkv, D).transpose(1, 2)
        return {"q": x[:, :H], "k": x[:, H:H + Hkv], "wq": 1 + 0.1 * rnd(D), "wk": 1 + 0.1 * rnd(D),
                "dq": rnd(B, H, S, D), "dk": rnd(B, Hkv, S, D)}
    if kind == "append":
        x = rnd(S, H + 2 * Hkv, D)
        page, pages = case["page"], case["pages"]
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:S].sort().values
        if S > 1:   # a padded step: rows without a slot
            slots = torch.where(torch.rand(S, generator=g, device="cuda") < 0.05, -1, slots)
        return {"q": x[:, :H], "k": x[:, H:H + Hkv], "v": x[:, H + Hkv:], "wq": 1 + 0.1 * rnd(D), "wk": 1 + 0.1 * rnd(D),
                "kc": rnd(pages, Hkv, page, D), "vc": rnd(pages, Hkv, page, D), "slots": slots,
                "positions": whole(0, 32768, S)}
    if kind in ("sinks", "prompt"):
        t = {"q": rnd(B, H, S, D), "k": rnd(B, Hkv, S, D), "v": rnd(B, Hkv, S, D)}
        if kind == "sinks":
            t["do"] = rnd(B, H, S, D)
        return t
    t = {"q": rnd(B, H, D)}
    if case["ragged"]:
        t["lens"] = whole(max(1, S // 4), S + 1, B)
    else:
        t["lens"] = torch.full((B,), S, dtype=torch.int32, device="cuda")
    if kind == "stream":
        t["k"], t["v"] = rnd(B, Hkv, S, D), rnd(B, Hkv, S, D)
        return t
    page = case["page"]
    n = -(-S // page)   # pages of a sequence, in any order in the pool, which has a few more
    t["k"], t["v"] = rnd(B * n + 3, Hkv, page, D), rnd(B * n + 3, Hkv, page, D)
    t["table"] = torch.randperm(B * n + 3, generator=g, device="cuda")[:B * n].to(torch.int32).reshape(B, n)
    return t


def prepare(case, seed):
    t = _tensors(case, seed)
    kind = case["kind"]
    state = {"case": case, "t": t, "kw": dict(rope=case["rope"], theta=case["theta"])}
    if kind == "qknorm":
        for n in ("q", "k", "wq", "wk"):
            t[n] = t[n].detach().requires_grad_(True)
    if kind == "sinks":
        for n in ("q", "k", "v"):
            t[n].requires_grad_(True)
    if kind in ("paged", "stream"):   # a server keeps its outputs
        state["buf"] = dict(out=torch.empty_like(t["q"]), lse=torch.empty(t["q"].shape[:2], dtype=torch.float32,
                                                                         device="cuda"))
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    with torch.set_grad_enabled(own and state["case"]["kind"] in ("qknorm", "sinks")):
        return _framework(state) if own else _PLAIN[state["case"]["kind"]](state["case"], state["t"])


def _framework(state):
    from paper_2609_13612_amd import api, autograd
    t, kw, case = state["t"], state["kw"], state["case"]
    kind = case["kind"]
    if kind == "qknorm":
        qr, kr = autograd.qknorm_rope(t["q"], t["k"], t["wq"], t["wk"], eps=EPS, **kw)
        return (qr.detach(), kr.detach()) + torch.autograd.grad((qr, kr), (t["q"], t["k"], t["wq"], t["wk"]),
                                                                (t["dq"], t["dk"]))
    if kind == "append":
        qr = api.attnfuse_qknorm_rope_append(t["q"], t["k"], t["v"], t["kc"], t["vc"], t["slots"], t["wq"], t["wk"], eps=EPS,
                                             positions=t["positions"], max_positions=32768, **kw)
        return qr, t["kc"], t["vc"]
    mask = dict(mask="sliding_window", window=case["W"], sinks=case["sinks"]) if case["W"] else dict(mask="causal")
    if kind == "sinks":
        o = autograd.attention(t["q"], t["k"], t["v"], **mask, **kw)
        return (o.detach(),) + torch.autograd.grad(o, (t["q"], t["k"], t["v"]), t["do"])
    if kind == "prompt":
        return api.attnfuse_fwd(t["q"], t["k"], t["v"], **mask, **kw)
    if kind == "stream":
        return api.attnfuse_decode(t["q"], t["k"], t["v"], t["lens"], **mask, **kw, **state["buf"])
    return api.attnfuse_decode_paged(t["q"], t["k"], t["v"], t["table"], t["lens"], **mask, **kw, **state["buf"])


# ---------------------------------------------------------------- the plain forms
def _rotate(x, pos, case, sign=1.0):
    """Rows of x [..., D] (fp32) rotated by sign * their positions' angles; pos broadcasts against x's rows."""
    if case["rope"] == "none":
        return x
    D = x.shape[-1]
    w = case["theta"] ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=x.device) / D)
    a = pos.double()[..., None] * w   # in 64 bits: far positions
    c, s = a.cos().float(), (sign * a.sin()).float()
    if case["rope"] == "neox":
        x0, x1 = x[..., : D // 2], x[..., D // 2:]
        return torch.cat((x0 * c - x1 * s, x0 * s + x1 * c), -1)
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack((x0 * c - x1 * s, x0 * s + x1 * c), -1).flatten(-2)


def _norm(x):
    """x (fp32) over the root of its mean square, and the factor."""
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_qknorm_one(x, w, dout, pos, case):
    x, w, dtype = x.float(), w.float(), x.dtype
    xh, r = _norm(x)
    out = _rotate(xh * w, pos, case)
    dy = _rotate(dout.float(), pos, case, -1.0)
    dw = (dy * xh).double().sum((0, 1, 2))
    g = dy * w
    return out.to(dtype), (r * (g - xh * (g * xh).mean(-1, keepdim=True))).to(dtype), dw.to(dtype)


def _plain_qknorm(case, t):
    pos = torch.arange(case["S"], device="cuda")
    qr, dq, dwq = _plain_qknorm_one(t["q"], t["wq"], t["dq"], pos, case)
    kr, dk, dwk = _plain_qknorm_one(t["k"], t["wk"], t["dk"], pos, case)
    return qr, kr, dq, dk, dwq, dwk


def _plain_append(case, t):
    pos = t["positions"][:, None]
    qr = _rotate(_norm(t["q"].float())[0] * t["wq"].float(), pos, case).to(t["q"].dtype)
    kr = _rotate(_norm(t["k"].float())[0] * t["wk"].float(), pos, case).to(t["q"].dtype)
    kept = t["slots"] >= 0
    at = t["slots"][kept]
    t["kc"].transpose(1, 2)[at // case["page"], at % case["page"]] = kr[kept]
    t["vc"].transpose(1, 2)[at // case["page"], at % case["page"]] = t["v"][kept]
    return qr, t["kc"], t["vc"]


def _band(x, W):
    """Blocks of W rows, each after the block before it: x [B, h, n W, D] -> [B, h, n, 2 W, D]."""
    B, h, S, D = x.shape
    x = x.reshape(B, h, S // W, W, D)
    before = torch.nn.functional.pad(x, (0, 0, 0, 0, 1, 0))[:, :, :-1]
    return torch.cat((before, x), 3)


def _plain_sinks(case, t):
    """In bands: queries in blocks of W, each against its own block of keys, the block before and the sinks."""
    B, H, Hkv, S, D = (case[k] for k in ("B", "H", "Hkv", "S", "D"))
    W, G, dtype, scale = min(case["W"], S), H // Hkv, t["q"].dtype, 1.0 / math.sqrt(D)
    n, ns = -(-S // W), min(case["sinks"], S)
    pos = torch.arange(S, device="cuda")

    def blocks(x):   # [B, H, S, D] -> [B, Hkv, n, G W, D], padded with zeros
        x = torch.nn.functional.pad(x, (0, 0, 0, n * W - S))
        return x.reshape(B, Hkv, G, n, W, D).transpose(2, 3).reshape(B, Hkv, n, G * W, D)

    def unblocks(x):
        return x.reshape(B, Hkv, n, G, W, -1).transpose(2, 3).reshape(B, H, n * W, -1)[:, :, :S]

    def keys(x):
        band = _band(torch.nn.functional.pad(x, (0, 0, 0, n * W - S)), W)
        return torch.cat((band, x[:, :, None, :ns].expand(B, Hkv, n, ns, D)), 3)

    def unkeys(x):   # each key's sum over the blocks that see it
        own_, before = x[..., W:2 * W, :], torch.nn.functional.pad(x[:, :, 1:, :W], (0, 0, 0, 0, 0, 1))
        y = (own_ + before).reshape(B, Hkv, n * W, D)[:, :, :S].clone()
        y[:, :, :ns] += x[..., 2 * W:, :].sum(2)
        return y

    q, k = blocks(_rotate(t["q"].float(), pos, case)), keys(_rotate(t["k"].float(), pos, case))
    v = keys(t["v"].float())
    b = torch.arange(n, device="cuda")[:, None, None]
    i = b * W + torch.arange(W, device="cuda")[None, :, None]
    j = (b - 1) * W + torch.arange(2 * W, device="cuda")[None, None, :]
    first = torch.arange(ns, device="cuda")[None, None, :].expand(n, W, ns)
    ok = torch.cat(((j >= 0) & (j <= i) & (j > i - W), first <= i - W), 2).repeat(1, G, 1)   # [n, G W, 2 W + ns]
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).masked_fill_(~ok, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    p.div_(l)
    o = torch.matmul(p, v)
    out = unblocks(o).to(dtype)
    if case["kind"] == "prompt":
        return out, unblocks(m + l.log())[..., 0]
    do = blocks(t["do"].float())
    dv = unkeys(torch.matmul(p.transpose(-1, -2), do))
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq = _rotate(unblocks(torch.matmul(ds, k)), pos, case, -1.0)
    dk = _rotate(unkeys(torch.matmul(ds.transpose(-1, -2), q)), pos, case, -1.0)
    return out, dq.to(dtype), dk.to(dtype), dv.to(dtype)


def _plain_decode(case, t, k, v):
    """One query per sequence against k, v [B, H_kv, n, D], of which lens are filled."""
    B, H, Hkv, D = (case[x] for x in ("B", "H", "Hkv", "D"))
    lens = t["lens"].long()
    q = _rotate(t["q"].float(), (lens - 1)[:, None], case).reshape(B, Hkv, H // Hkv, D)
    j = torch.arange(k.shape[2], device="cuda")[None, :]
    ok = j < lens[:, None]
    if case["W"]:
        ok = ok & ((j >= lens[:, None] - case["W"]) | (j < case["sinks"]))
    s = torch.matmul(q, k.float().transpose(-1, -2)).mul_(1.0 / math.sqrt(D)).masked_fill_(~ok[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    return (torch.matmul(p, v.float()) / l).reshape(B, H, D).to(t["q"].dtype), (m + l.log()).reshape(B, H)


def _gathered(cache, table):
    """The pages of every sequence in order: [B, H_kv, pages * page, D]."""
    x = cache[table.long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])


def _plain_paged(case, t):
    return _plain_decode(case, t, _gathered(t["k"], t["table"]), _gathered(t["v"], t["table"]))


def _plain_stream(case, t):
    return _plain_decode(case, t, t["k"], t["v"])


_PLAIN = {"qknorm": _plain_qknorm, "append": _plain_append, "sinks": _plain_sinks, "prompt": _plain_sinks,
          "paged": _plain_paged, "stream": _plain_stream}


# ---------------------------------------------------------------- what a pass cannot do without
def _pairs(S, W, sinks):
    """Visible (query, key) pairs of one head."""
    w, far = min(W, S), max(0, S - W)   # rows past the window see the sinks that have left it too
    band = w * (w + 1) // 2 + far * w
    m = min(sinks, far)
    return band + m * (m + 1) // 2 + (far - m) * m


def work(case):
    B, H, Hkv, S, D, kind = (case[k] for k in ("B", "H", "Hkv", "S", "D", "kind"))
    es = 4 if case["dtype"] == "fp32" else 2
    qn, kn = B * H * S * D, B * Hkv * S * D
    if kind == "qknorm":   # x and the gradient in, the rotated rows and the gradient out
        return {"bytes": 4 * es * (qn + kn), "flops": 24 * (qn + kn)}
    if kind == "append":   # 5 % of the rows have no slot
        return {"bytes": es * 2 * (qn + 2 * kn) + 12 * S, "flops": 9 * (qn + kn)}
    if kind in ("sinks", "prompt"):
        pairs = B * H * _pairs(S, case["W"], case["sinks"])
        if kind == "prompt":
            return {"bytes": es * (2 * qn + 2 * kn) + 4 * B * H * S, "flops": 4 * D * pairs}
        return {"bytes": es * (4 * qn + 4 * kn), "flops": 14 * D * pairs}
    n = S * 5 // 8 if case["ragged"] else S   # lengths are uniform over [S / 4, S]
    if case["W"]:
        n = min(n, case["W"] + case["sinks"])
    return {"bytes": es * (2 * B * Hkv * n * D + 2 * B * H * D) + 4 * B * H + 4 * B, "flops": 4 * D * B * H * n}


# ---------------------------------------------------------------- the same in 64 bits, from the definition
def exact(case, seed):
    with torch.no_grad():
        return getattr(_Exact, case["kind"])(case, _tensors(case, seed))


class _Exact:
    """Every kind's outputs, a head at a time."""

    @staticmethod
    def turn(x, pos, case, back=False):
        """Row n of x [n, D] turned by the angles of pos[n], its pairs as complex numbers."""
        if case["rope"] == "none":
            return x
        D = x.shape[-1]
        half = torch.arange(D // 2, device=x.device)
        a, b = (half, half + D // 2) if case["rope"] == "neox" else (2 * half, 2 * half + 1)
        angle = pos.double()[:, None] * torch.exp(half.double() * (-2.0 / D * math.log(case["theta"])))
        z = torch.complex(x[:, a], x[:, b]) * torch.polar(torch.ones_like(angle), -angle if back else angle)
        y = torch.empty_like(x)
        y[:, a], y[:, b] = z.real, z.imag
        return y

    @staticmethod
    def size(row):
        return (row.pow(2).sum(1, keepdim=True) / row.shape[1] + EPS).sqrt()

    @staticmethod
    def qknorm(case, t):
        D, pos, got = case["D"], torch.arange(case["S"], device="cuda"), []
        for x, w, dout in ((t["q"], t["wq"], t["dq"]), (t["k"], t["wk"], t["dk"])):
            w = w.double()
            out, dx = (torch.empty(x.shape, dtype=torch.float64, device="cuda") for _ in range(2))
            dw = torch.zeros_like(w)
            for b in range(x.shape[0]):
                for h in range(x.shape[1]):
                    row, dy = x[b, h].double(), _Exact.turn(dout[b, h].double(), pos, case, back=True)
                    size = _Exact.size(row)
                    out[b, h] = _Exact.turn(row / size * w, pos, case)
                    dw += (dy * row / size).sum(0)
                    dx[b, h] = dy * w / size - row * ((dy * w * row).sum(1, keepdim=True) / (D * size.pow(3)))
            got.append((out, dx, dw))
        return tuple(got[n][i] for i in range(3) for n in range(2))

    @staticmethod
    def append(case, t):
        page, pos, got = case["page"], t["positions"], []
        for x, w in ((t["q"], t["wq"]), (t["k"], t["wk"])):
            out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            for h in range(x.shape[1]):
                row = x[:, h].double()
                out[:, h] = _Exact.turn(row / _Exact.size(row) * w.double(), pos, case)
            got.append(out)
        kc, vc = t["kc"].double(), t["vc"].double()
        rows = (t["slots"] >= 0).nonzero()[:, 0]
        page_of, at = t["slots"][rows] // page, t["slots"][rows] % page
        for h in range(case["Hkv"]):
            kc[page_of, h, at] = got[1][rows, h]
            vc[page_of, h, at] = t["v"][rows, h].double()
        return got[0], kc, vc

    @staticmethod
    def sinks(case, t):
        B, H, Hkv, S, D = (case[k] for k in ("B", "H", "Hkv", "S", "D"))
        pos, train = torch.arange(S, device="cuda"), case["kind"] == "sinks"
        o, lse = torch.empty(B, H, S, D, dtype=torch.float64, device="cuda"), torch.empty(B, H, S, dtype=torch.float64)
        dq, dk, dv = (torch.zeros(B, h if train else 0, S, D, dtype=torch.float64, device="cuda") for h in (H, Hkv, Hkv))
        far = pos[:, None] - pos[None, :]
        hidden = (far < 0) | ((far >= case["W"]) & (pos[None, :] >= case["sinks"]))
        for b in range(B):
            for h in range(H):
                g = h // (H // Hkv)
                q, k = _Exact.turn(t["q"][b, h].double(), pos, case), _Exact.turn(t["k"][b, g].double(), pos, case)
                v = t["v"][b, g].double()
                s = (q @ k.T).div_(math.sqrt(D)).masked_fill_(hidden, -math.inf)
                lse[b, h] = torch.logsumexp(s, 1).cpu()
                p = torch.softmax(s, 1)
                del s
                o[b, h] = p @ v
                if train:
                    do = t["do"][b, h].double()
                    dp = do @ v.T
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(D)
                    dv[b, g] += p.T @ do
                    dq[b, h] = _Exact.turn(ds @ k, pos, case, back=True)
                    dk[b, g] += _Exact.turn(ds.T @ q, pos, case, back=True)
        return (o, dq, dk, dv) if train else (o, lse)

    prompt = sinks

    @staticmethod
    def paged(case, t):
        B, H, Hkv, D = (case[k] for k in ("B", "H", "Hkv", "D"))
        o, lse = torch.empty(B, H, D, dtype=torch.float64), torch.empty(B, H, dtype=torch.float64)
        for b, n in enumerate(t["lens"].tolist()):
            at = torch.arange(n, device="cuda")
            if case["W"]:
                at = at[(at >= n - case["W"]) | (at < case["sinks"])]
            q = _Exact.turn(t["q"][b].double(), torch.full((H,), n - 1, device="cuda"), case)
            for g in range(Hkv):
                if case["kind"] == "paged":
                    pages = t["table"][b].long()[at // case["page"]]
                    k, v = (t[x][pages, g, at % case["page"]].double() for x in ("k", "v"))
                else:
                    k, v = (t[x][b, g, at].double() for x in ("k", "v"))
                heads = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
                s = q[heads] @ k.T / math.sqrt(D)
                lse[b, heads] = torch.logsumexp(s, 1).cpu()
                o[b, heads] = (torch.softmax(s, 1) @ v).cpu()
        return o, lse

    stream = paged
