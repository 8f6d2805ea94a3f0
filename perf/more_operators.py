"""The calls that the operators for images, video and shared prefixes are measured on, over the ranges their users meet.

Kinds of call, each through a public entry point:

  rotate   autograd.qknorm_rope with positions of several axes, forward and backward, as a layer is trained: the per-head
           RMS norm of queries and keys and their rotation, or the rotation alone; q and k are views of the fused
           projection's output [B, S, (H + 2 H_kv) D]
  append   api.attnfuse_qknorm_rope_append with positions of several axes: new tokens, keys and values written to pages
  decode   api.attnfuse_decode_paged with a prefix that the batch shares: one new token per sequence
  prompts  api.attnfuse_fwd_paged: several new tokens per sequence against its pages, behind a shared prefix or without

Each has its plain form here, in elementary torch operations.  Tensors are N(0, 1), as in the framework's parity
workloads, and norm weights 1 + N(0, 0.1); positions are those of a text, frames of patches and a text behind them.
"""
import math
import random

import torch

own = False

HEADS = ((32, 8, 128), (64, 8, 128), (16, 16, 128), (12, 12, 64), (16, 16, 64), (8, 2, 64), (12, 4, 128))
SECTIONS = {64: ((16, 16), (8, 12, 12), (10, 11, 11), (5, 27), (8, 8, 8, 8)),
            128: ((32, 32), (16, 24, 24), (24, 20, 20), (7, 28, 29), (16, 16, 16, 16))}
EPS = 1e-6
MAX_POSITION = 32768


def _case(kind, **kw):
    c = dict(kind=kind, B=1, H=32, Hkv=8, D=128, dtype="bf16")
    if kind in ("rotate", "append"):
        c.update(S=8192, rope="neox", theta=500000.0, sections="16,24,24", order="blocks", ladder="shared", norm=True)
    else:
        c.update(P=0, ctx=0, page=64)
    c.update(kw)
    return c


def listed():
    return [
        # Queries and keys of a Llama-3-8B layer trained on a text with a video: time, height and width.
        _case("rotate", name="rotate_video_8k"),
        # GPT-2-small heads over patches of images: two axes with a ladder of frequencies each, no norm, odd length.
        _case("rotate", name="rotate_image_d64", B=4, H=12, Hkv=12, S=1777, D=64, rope="interleaved", theta=10000.0,
              sections="16,16", ladder="own", norm=False),
        # The fp32 arithmetic that a port is checked with; axes in turns.
        _case("rotate", name="rotate_turns_fp32", B=2, H=8, Hkv=2, S=777, sections="24,20,20", order="turns", dtype="fp32"),
        # One sequence's newest token: the smallest call that a server makes per layer.
        _case("append", name="append_axes_one", S=1, pages=512, page=16),
        # A step's mixed batch: frames of videos and single tokens, some rows padding, into pages of 64.
        _case("append", name="append_axes_frames", S=4500, H=64, pages=1200, page=64, order="turns", norm=False),
        # A few chats behind a short system prompt: latency.
        _case("decode", name="decode_shared_small", B=4, P=500, ctx=60, page=16),
        # A batch of questions about one long text: the prefix's bytes are what has to be read.
        _case("decode", name="decode_shared_32k", B=32, P=32768, ctx=1024),
        # Many samples of one prompt, Llama-3-70B heads: the prefix's products count.
        _case("decode", name="decode_shared_many", B=256, H=64, P=8192, ctx=512),
        # Small heads, one to a group, odd lengths in small pages.
        _case("decode", name="decode_shared_d64", B=24, H=12, Hkv=12, D=64, P=5001, ctx=300, page=16),
        # Questions of some tokens each about one video.
        _case("prompts", name="prompts_questions", B=24, n=60, P=16384, ctx=40),
        # Chunks of long prompts without a prefix, in a batch padded for a captured graph.
        _case("prompts", name="prompts_chunks", B=4, n=512, ctx=16384, pad=100),
        # Long documents behind a long shared prefix: the most work.
        _case("prompts", name="prompts_long", B=6, n=1000, P=32768, ctx=2000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rotate", "rotate", "append", "decode", "decode", "prompts", "prompts"))
    H, Hkv, D = rng.choice(HEADS)
    v = dict(H=H, Hkv=Hkv, D=D)
    if kind in ("rotate", "append"):
        v.update(rope=rng.choice(("neox", "neox", "interleaved")), theta=rng.choice((10000.0, 500000.0)),
                 sections=",".join(map(str, rng.choice(SECTIONS[D]))), order=rng.choice(("blocks", "turns")),
                 ladder=rng.choice(("shared", "shared", "own")), norm=rng.random() < 0.6,
                 dtype=rng.choice(("bf16", "bf16", "fp32")))
        if kind == "rotate":
            S = _log(rng, 5, 8192)
            return _case(kind, B=max(1, min(rng.randint(1, 6), 8192 // S)), S=S, **v)
        T, page = _log(rng, 1, 4500), rng.choice((16, 32, 64, 128, 256))
        return _case(kind, S=T, page=page, pages=2 + 2 * T // page + rng.randint(0, 64), **v)
    page = rng.choice((16, 16, 32, 64, 128, 256))
    P = _log(rng, 20, 32768)
    if kind == "decode":
        B = max(1, min(_log(rng, 1, 256), 256 * 8192 // P))
        return _case(kind, B=B, P=P, ctx=max(1, min(_log(rng, 1, 4096), 160 * 1024 // B)), page=page, **v)
    P = P if rng.random() < 0.7 else 0
    n, ctx = _log(rng, 1, 1000), _log(rng, 1, 16384)
    B = max(1, min(_log(rng, 1, 48), 128000 // (n * H), 128 * 1024 // ctx))
    return _case(kind, B=B, n=n, P=P, ctx=ctx, page=page, pad=rng.choice((0, 0, 3, 50)), **v)


# ---------------------------------------------------------------- inputs
def _sections(case):
    return tuple(int(s) for s in case["sections"].split(","))


def _spread(case):
    """Queries and own keys of every sequence of a batch, from the case's sizes alone."""
    rng = random.Random(case["B"] * 1000003 + case["P"] * 1009 + case["ctx"])
    n = case.get("n", 1)
    queries = [rng.randint(max(1, n // 4), n) for _ in range(case["B"])]
    return queries, [m + rng.randint(case["ctx"] // 4, case["ctx"]) for m in queries]


def _positions(case, lead, g):
    """int32 [axes, *lead, S]: a text, frames of patches and a text behind them, each batch from a start of its own."""
    S, axes = case["S"], len(_sections(case))
    side = max(1, int(math.sqrt(S) / 2))
    text = S // 8
    i = torch.arange(S, device="cuda")
    j = (i - text).clamp(min=0)
    frame, row, col = j // (side * side), j // side % side, j % side
    grid = {2: (row, col), 3: (frame, row, col), 4: (frame // 4, frame % 4, row, col)}[axes]
    behind = S - S // 8
    last = text + S // (side * side) + side
    p = torch.stack([torch.where(i < text, i, torch.where(i < behind, text + a, last + i - behind)) for a in grid])
    start = torch.randint(0, MAX_POSITION - 2 * S - 64, lead, generator=g, device="cuda")
    return (p.reshape(axes, *(1 for _ in lead), S) + start[None, ..., None]).to(torch.int32)


def _tensors(case, seed):
    """The tensors of a case, on the GPU, from the seed alone."""
    g = torch.Generator("cuda").manual_seed(seed)
    B, H, Hkv, D, kind = (case[k] for k in ("B", "H", "Hkv", "D", "kind"))
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16

    def rnd(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    if kind in ("rotate", "append"):
        S = case["S"]
        t = {"wq": 1 + 0.1 * rnd(D), "wk": 1 + 0.1 * rnd(D)} if case["norm"] else {"wq": None, "wk": None}
        if kind == "rotate":
            x = rnd(B, S, H + 2 * Hkv, D).transpose(1, 2)
            t.update(q=x[:, :H], k=x[:, H:H + Hkv], dq=rnd(B, H, S, D), dk=rnd(B, Hkv, S, D), pos=_positions(case, (B,), g))
            return t
        x = rnd(S, H + 2 * Hkv, D)
        page, pages = case["page"], case["pages"]
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:S].sort().values
        if S > 1:   # a padded step: rows without a slot
            slots = torch.where(torch.rand(S, generator=g, device="cuda") < 0.05, -1, slots)
        t.update(q=x[:, :H], k=x[:, H:H + Hkv], v=x[:, H + Hkv:], kc=rnd(pages, Hkv, page, D), vc=rnd(pages, Hkv, page, D),
                 slots=slots, pos=_positions(case, (), g))
        return t
    queries, lens = _spread(case)
    page, P = case["page"], case["P"]
    width, ahead = -(-max(lens) // page), -(-P // page)
    pages = B * width + ahead + 3   # in any order in the pool, which has a few more
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    tokens = sum(queries) + case.get("pad", 0)
    t = {"q": rnd(tokens, H, D), "k": rnd(pages, Hkv, page, D), "v": rnd(pages, Hkv, page, D),
         "table": order[:B * width].reshape(B, width), "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "prefix": order[B * width:B * width + ahead] if P else None,
         "plen": torch.tensor([P], dtype=torch.int32, device="cuda") if P else None}
    starts = [sum(queries[:b]) for b in range(B + 1)]
    t["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    t["host"] = list(zip(starts, queries, lens))
    return t


def prepare(case, seed):
    t = _tensors(case, seed)
    state = {"case": case, "t": t}
    if case["kind"] == "rotate":
        for n in ("q", "k", "wq", "wk"):
            if t[n] is not None:
                t[n] = t[n].detach().requires_grad_(True)
    if case["kind"] in ("decode", "prompts"):   # a server keeps its outputs
        state["buf"] = dict(out=torch.zeros_like(t["q"]), lse=torch.zeros(t["q"].shape[:2], dtype=torch.float32,
                                                                         device="cuda"))
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    with torch.set_grad_enabled(own and state["case"]["kind"] == "rotate"):
        return _framework(state) if own else _PLAIN[state["case"]["kind"]](state["case"], state["t"])


def _framework(state):
    from paper_2609_13612_amd import api, autograd
    t, case = state["t"], state["case"]
    kind = case["kind"]
    if kind in ("rotate", "append"):
        kw = dict(rope=case["rope"], theta=case["theta"], positions=t["pos"], max_positions=MAX_POSITION,
                  sections=_sections(case), section_order=case["order"], frequencies=case["ladder"], norm=case["norm"], eps=EPS)
        if kind == "append":
            qr = api.attnfuse_qknorm_rope_append(t["q"], t["k"], t["v"], t["kc"], t["vc"], t["slots"], t["wq"], t["wk"], **kw)
            return qr, t["kc"], t["vc"]
        qr, kr = autograd.qknorm_rope(t["q"], t["k"], t["wq"], t["wk"], **kw)
        leaves = [t[n] for n in ("q", "k", "wq", "wk") if t[n] is not None]
        return (qr.detach(), kr.detach()) + torch.autograd.grad((qr, kr), leaves, (t["dq"], t["dk"]))
    prefix = dict(prefix_table=t["prefix"], prefix_len=t["plen"])
    if kind == "decode":
        return api.attnfuse_decode_paged(t["q"], t["k"], t["v"], t["table"], t["lens"], **prefix, **state["buf"])
    return api.attnfuse_fwd_paged(t["q"], t["k"], t["v"], t["table"], t["starts"], t["lens"], **prefix, **state["buf"])


# ---------------------------------------------------------------- the plain forms
def _axis_and_rung(case):
    """For every pair: its axis, and theta's exponent in its frequency."""
    s, half = _sections(case), case["D"] // 2
    if case["order"] == "blocks":
        axis = [a for a, n in enumerate(s) for _ in range(n)]
    else:
        axis = [a for r in range(max(s)) for a, n in enumerate(s) if n > r]
    if case["ladder"] == "shared":
        return axis, [-i / half for i in range(half)]
    return axis, [-axis[:i].count(axis[i]) / s[axis[i]] for i in range(half)]


def _cos_sin(pos, case):
    """cos and sin [..., D / 2] of the angles of positions [axes, ...]."""
    axis, rung = _axis_and_rung(case)
    w = case["theta"] ** torch.tensor(rung, dtype=torch.float64, device=pos.device)
    a = pos.double()[axis].movedim(0, -1) * w   # in 64 bits: far positions
    return a.cos().float(), a.sin().float()


def _rotate(x, c, s, case):
    D = x.shape[-1]
    if case["rope"] == "neox":
        x0, x1 = x[..., : D // 2], x[..., D // 2:]
        return torch.cat((x0 * c - x1 * s, x0 * s + x1 * c), -1)
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack((x0 * c - x1 * s, x0 * s + x1 * c), -1).flatten(-2)


def _plain_rotate(case, t):
    c, s = _cos_sin(t["pos"][:, :, None], case)
    out, dx, dw = [], [], []
    for x, w, dout in ((t["q"], t["wq"], t["dq"]), (t["k"], t["wk"], t["dk"])):
        dtype, x, g = x.dtype, x.float(), _rotate(dout.float(), c, -s, case)
        if w is None:
            out.append(_rotate(x, c, s, case).to(dtype))
            dx.append(g.to(dtype))
            continue
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        x = x * r
        out.append(_rotate(x * w.float(), c, s, case).to(dtype))
        dw.append((g * x).double().sum((0, 1, 2)).to(dtype))
        g = g * w.float()
        dx.append((r * (g - x * (g * x).mean(-1, keepdim=True))).to(dtype))
    return (*out, *dx, *dw)


def _plain_append(case, t):
    c, s = _cos_sin(t["pos"][:, :, None], case)
    got = []
    for x, w in ((t["q"], t["wq"]), (t["k"], t["wk"])):
        dtype, x = x.dtype, x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
        got.append(_rotate(x, c, s, case).to(dtype))
    kept = t["slots"] >= 0
    at = t["slots"][kept]
    t["kc"].transpose(1, 2)[at // case["page"], at % case["page"]] = got[1][kept]
    t["vc"].transpose(1, 2)[at // case["page"], at % case["page"]] = t["v"][kept]
    return got[0], t["kc"], t["vc"]


def _gathered(cache, pages, n):
    """The first n keys of a list of pages, in order, as fp32: [..., H_kv, n, D]."""
    x = cache[pages.long()].transpose(-4, -3)
    return x.reshape(*x.shape[:-3], -1, x.shape[-1])[..., :n, :].float()


def _softmax_stats(s):
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    return p.div_(l), (m + l.log())[..., 0]


def _plain_decode(case, t):
    """The prefix's scores of the whole batch in one product, each sequence's own behind them."""
    B, H, Hkv, D, P = (case[x] for x in ("B", "H", "Hkv", "D", "P"))
    q, scale = t["q"].float().reshape(B, Hkv, H // Hkv, D), 1.0 / math.sqrt(D)
    n = t["table"].shape[1] * case["page"]
    k0, v0 = _gathered(t["k"], t["prefix"], P), _gathered(t["v"], t["prefix"], P)
    k1, v1 = _gathered(t["k"], t["table"], n), _gathered(t["v"], t["table"], n)
    rows = q.transpose(0, 1).reshape(Hkv, -1, D)
    s0 = torch.matmul(rows, k0.transpose(-1, -2)).reshape(Hkv, B, H // Hkv, P).transpose(0, 1)
    ok = torch.arange(n, device="cuda") < t["lens"][:, None]
    s1 = torch.matmul(q, k1.transpose(-1, -2)).masked_fill_(~ok[:, None, None], -math.inf)
    p, lse = _softmax_stats(torch.cat((s0, s1), -1).mul_(scale))
    o = torch.matmul(p[..., :P].transpose(0, 1).reshape(Hkv, -1, P), v0).reshape(Hkv, B, H // Hkv, D).transpose(0, 1)
    o = o + torch.matmul(p[..., P:], v1)
    return o.reshape(B, H, D).to(t["q"].dtype), lse.reshape(B, H)


def _plain_prompts(case, t):
    H, Hkv, D, P = (case[x] for x in ("H", "Hkv", "D", "P"))
    G, scale = H // Hkv, 1.0 / math.sqrt(D)
    out, lse = torch.zeros_like(t["q"]), torch.zeros(t["q"].shape[:2], dtype=torch.float32, device="cuda")
    if P:
        k0, v0 = _gathered(t["k"], t["prefix"], P), _gathered(t["v"], t["prefix"], P)
    for b, (start, n, keys) in enumerate(t["host"]):
        k, v = _gathered(t["k"], t["table"][b], keys), _gathered(t["v"], t["table"][b], keys)
        if P:
            k, v = torch.cat((k0, k), 1), torch.cat((v0, v), 1)
        q = t["q"][start:start + n].float().reshape(n, Hkv, G, D).transpose(0, 1).reshape(Hkv, n * G, D)
        s = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).reshape(Hkv, n, G, P + keys)
        late = torch.arange(keys, device="cuda") > keys - n + torch.arange(n, device="cuda")[:, None]
        s[..., P:].masked_fill_(late[None, :, None], -math.inf)
        p, stat = _softmax_stats(s)
        o = torch.matmul(p.reshape(Hkv, n * G, P + keys), v)
        out[start:start + n] = o.reshape(Hkv, n, G, D).transpose(0, 1).reshape(n, H, D).to(out.dtype)
        lse[start:start + n] = stat.transpose(0, 1).reshape(n, H)
    return out, lse


_PLAIN = {"rotate": _plain_rotate, "append": _plain_append, "decode": _plain_decode, "prompts": _plain_prompts}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    H, Hkv, D, kind = (case[k] for k in ("H", "Hkv", "D", "kind"))
    es = 4 if case["dtype"] == "fp32" else 2
    if kind in ("rotate", "append"):
        rows, axes = case["B"] * case["S"], len(_sections(case))
        qn, kn = rows * H * D, rows * Hkv * D
        if kind == "append":
            return {"bytes": es * 2 * (qn + 2 * kn) + (8 + 4 * axes) * rows, "flops": (9 if case["norm"] else 4) * (qn + kn)}
        # the rows and the gradients of the turned rows in, the turned rows and the rows' gradients out
        return {"bytes": 4 * es * (qn + kn) + 4 * axes * rows, "flops": (24 if case["norm"] else 8) * (qn + kn)}
    queries, lens = _spread(case)
    tokens, P = sum(queries), case["P"]
    pairs = sum(n * P + n * keys - n * (n - 1) // 2 for n, keys in zip(queries, lens))
    return {"bytes": es * 2 * (P + sum(lens)) * Hkv * D + es * 2 * tokens * H * D + 4 * tokens * H, "flops": 4 * D * H * pairs}


# ---------------------------------------------------------------- the same in 64 bits, from the definition
def exact(case, seed):
    with torch.no_grad():
        t = _tensors(case, seed)
        return getattr(_Exact, case["kind"])(case, t)


class _Exact:
    """Every kind's outputs, a head at a time."""

    @staticmethod
    def turns(case, pos):
        """The unit numbers [rows, D / 2] that the pairs of rows at positions [axes, rows] are multiplied by."""
        sections, half = _sections(case), case["D"] // 2
        left, angles = list(sections), []
        a = 0
        for i in range(half):
            if case["order"] == "blocks":
                while left[a] == 0:
                    a += 1
            else:   # the next axis, in a circle, that has pairs left
                a = a if i == 0 else (a + 1) % len(left)
                while left[a] == 0:
                    a = (a + 1) % len(left)
            rung = 2 * i / case["D"] if case["ladder"] == "shared" else (sections[a] - left[a]) / sections[a]
            left[a] -= 1
            angles.append(pos[a].double() * math.exp(-rung * math.log(case["theta"])))
        angle = torch.stack(angles, 1)
        return torch.polar(torch.ones_like(angle), angle)

    @staticmethod
    def turn(x, z, case):
        """Row n of x [n, D], its pairs as complex numbers, times z[n]."""
        D = x.shape[-1]
        half = torch.arange(D // 2, device=x.device)
        a, b = (half, half + D // 2) if case["rope"] == "neox" else (2 * half, 2 * half + 1)
        w = torch.complex(x[:, a], x[:, b]) * z
        y = torch.empty_like(x)
        y[:, a], y[:, b] = w.real, w.imag
        return y

    @staticmethod
    def size(row):
        return (row.pow(2).sum(1, keepdim=True) / row.shape[1] + EPS).sqrt()

    @staticmethod
    def rotate(case, t):
        D, outs, grads, weights = case["D"], [], [], []
        for x, w, dout in ((t["q"], t["wq"], t["dq"]), (t["k"], t["wk"], t["dk"])):
            out, dx = (torch.empty(x.shape, dtype=torch.float64, device="cuda") for _ in range(2))
            dw = torch.zeros(D, dtype=torch.float64, device="cuda")
            for b in range(x.shape[0]):
                z = _Exact.turns(case, t["pos"][:, b])
                for h in range(x.shape[1]):
                    row, dy = x[b, h].double(), _Exact.turn(dout[b, h].double(), z.conj(), case)
                    if w is None:
                        out[b, h], dx[b, h] = _Exact.turn(row, z, case), dy
                        continue
                    size, wd = _Exact.size(row), w.double()
                    out[b, h] = _Exact.turn(row / size * wd, z, case)
                    dw += (dy * row / size).sum(0)
                    dx[b, h] = dy * wd / size - row * ((dy * wd * row).sum(1, keepdim=True) / (D * size.pow(3)))
            outs.append(out)
            grads.append(dx)
            if w is not None:
                weights.append(dw)
        return (*outs, *grads, *weights)

    @staticmethod
    def append(case, t):
        page, z, got = case["page"], _Exact.turns(case, t["pos"]), []
        for x, w in ((t["q"], t["wq"]), (t["k"], t["wk"])):
            out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            for h in range(x.shape[1]):
                row = x[:, h].double()
                out[:, h] = _Exact.turn(row if w is None else row / _Exact.size(row) * w.double(), z, case)
            got.append(out)
        kc, vc = t["kc"].double(), t["vc"].double()
        rows = (t["slots"] >= 0).nonzero()[:, 0]
        page_of, at = t["slots"][rows] // page, t["slots"][rows] % page
        for h in range(case["Hkv"]):
            kc[page_of, h, at] = got[1][rows, h]
            vc[page_of, h, at] = t["v"][rows, h].double()
        return got[0], kc, vc

    @staticmethod
    def prompts(case, t):
        H, G, D, P, page = case["H"], case["H"] // case["Hkv"], case["D"], case["P"], case["page"]
        o = torch.zeros(t["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(t["q"].shape[:2], dtype=torch.float64, device="cuda")
        ahead = torch.arange(P, device="cuda")
        for b, (start, n, keys) in enumerate(t["host"]):
            at = torch.arange(keys, device="cuda")
            places = [t["table"][b].long()[at // page] * page + at % page]
            if P:
                places.insert(0, t["prefix"].long()[ahead // page] * page + ahead % page)
            places = torch.cat(places)
            last = P + keys - n + torch.arange(n, device="cuda")   # the last key that each query sees
            hidden = torch.arange(P + keys, device="cuda")[None] > last[:, None]
            for g in range(case["Hkv"]):
                k, v = (t[x][places // page, g, places % page].double() for x in ("k", "v"))
                for h in range(g * G, (g + 1) * G):
                    s = (t["q"][start:start + n, h].double() @ k.T).div_(math.sqrt(D)).masked_fill_(hidden, -math.inf)
                    lse[start:start + n, h] = torch.logsumexp(s, 1)
                    o[start:start + n, h] = torch.softmax(s, 1) @ v
        return o, lse

    decode = prompts
