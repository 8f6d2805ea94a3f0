"""Decode over a paged cache, and over a contiguous one with sinks, against the definition in 64 bits.

Tolerances.  P is rounded to bf16 before it meets V, and O on its way out: half a step (2^-8) of p |v| summed, and of O.  The
rotated query is kept to 2^-16 of itself and D products of it are summed in fp32 (2 D 2^-24 <= 2^-16 of their magnitudes), so
a score moves by at most 2^-15 of A = scale sum |q' k| (ALiBi's term adds its own to A), an LSE by as much, and a weight p by
twice that of itself; exp2, log2 and fp32 sums of thousands of weights add 2^-16 of p and 2^-18 (1 + |LSE|).
"""
import pytest
import torch

from gpu_util import announce, need_gpu
from llm_ref import assert_within, decode, f64, half_step
from paper_2609_13612_amd import api, inputs

pytestmark = pytest.mark.gpu
HALF = half_step(torch.bfloat16)


def seen_of(L, S, window, sinks):
    L = max(0, min(L, S))
    n = torch.arange(L)
    return n[(n >= L - window) | (n < sinks)] if window else n


def check(o, lse, refs, what):
    for b, (O, L, pv, mag) in enumerate(refs):
        tol = 2.0 ** -15 * mag
        assert_within(o[b], O, HALF * O.abs() + (HALF + 2 * tol[:, None] + 2.0 ** -16) * pv, f"{what} O[{b}]")
        fin = torch.isfinite(L)
        assert torch.equal(torch.isneginf(f64(lse[b])), ~fin), f"{what} LSE[{b}]"
        assert_within(lse[b].cpu()[fin], L[fin], (tol + 2.0 ** -18 * (1 + L.abs()))[fin], f"{what} LSE[{b}]")


def cache(B, Hkv, S, D, page, g, nhd=False, spare=2):
    """Pages in a random order with some to spare, the block table, and each sequence's keys and values in order."""
    n = -(-S // page)
    shape = (B * n + spare, page, Hkv, D) if nhd else (B * n + spare, Hkv, page, D)
    k, v = (torch.randn(shape, generator=g).bfloat16().cuda() for _ in "kv")
    if nhd:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    table = torch.randperm(B * n + spare, generator=g)[: B * n].reshape(B, n)
    flat = [[x.cpu()[table[b]].transpose(0, 1).reshape(Hkv, n * page, D) for x in (k, v)] for b in range(B)]
    return k, v, table.to(torch.int32).cuda(), flat


CASES = [
    # B, H, Hkv, S, D, page, lens, rope, window, sinks, alibi, places first
    (1, 32, 8, 4096, 128, 16, [4096], "neox", 0, 0, False, False),
    (1, 2, 1, 16, 64, 16, [1], "none", 0, 0, False, False),
    (5, 8, 2, 700, 64, 16, [700, 0, -3, 9999, 33], "interleaved", 0, 0, False, True),
    (3, 12, 12, 1000, 64, 32, [999, 512, 31], "none", 0, 0, True, False),
    (4, 64, 8, 2000, 128, 64, [2000, 1, 17, 1025], "neox", 100, 4, False, False),
    (3, 6, 2, 5000, 128, 256, [5000, 4097, 40], "interleaved", 1000, 300, False, True),
    (2, 40, 1, 300, 128, 16, [300, 77], "neox", 0, 0, False, False),           # 40 heads: two groups
    (2, 33, 1, 300, 64, 128, [300, 129], "none", 64, 0, True, False),
    (70, 4, 1, 900, 128, 16, [(37 * i) % 901 for i in range(70)], "neox", 50, 20, False, False),
    (1, 3, 3, 20000, 64, 16, [19999], "neox", 0, 0, False, False),
    (2, 4, 4, 600, 128, 16, [600, 555], "neox", 1, 1, False, False),
    (2, 4, 4, 600, 128, 16, [600, 555], "none", 5000, 7, False, False),        # a window over everything
    (2, 4, 2, 640, 64, 64, [600, 555], "none", 40, 5000, False, False),        # sinks over everything
    (1, 8, 1, 200, 128, 1024, [190], "neox", 0, 0, False, False),              # a page longer than the sequence
]


@pytest.mark.parametrize("B,H,Hkv,S,D,page,lens,rope,window,sinks,alibi,nhd", CASES, ids=lambda x: str(x)[:18])
def test_paged(B, H, Hkv, S, D, page, lens, rope, window, sinks, alibi, nhd):
    need_gpu()
    announce(f"paged B={B} H={H}/{Hkv} S={S} D={D} page={page} {rope} W={window} sinks={sinks} alibi={alibi} nhd={nhd}")
    g = torch.Generator().manual_seed(S + page)
    k, v, table, flat = cache(B, Hkv, S, D, page, g, nhd)
    q = torch.randn(B, H, D, generator=g).bfloat16().cuda()
    slopes = inputs.alibi_slopes(H) if alibi else None
    mask = dict(mask="sliding_window", window=window, sinks=sinks) if window else dict(mask="causal")
    most = table.shape[1] * page
    nbytes = api.attnfuse_decode_paged_workspace_bytes(B, H, Hkv, most, D, window, sinks)
    guard = torch.full((nbytes + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    o, lse = api.attnfuse_decode_paged(q, k, v, table, torch.tensor(lens, dtype=torch.int32).cuda(), rope=rope,
                                       theta=500000.0, alibi_slopes=None if slopes is None else slopes.cuda(),
                                       workspace=guard[:nbytes], **mask)
    torch.cuda.synchronize()
    assert (guard[nbytes:] == 0x5A).all(), "written past the workspace"
    refs = [decode(q[b], *flat[b], seen_of(lens[b], most, window, sinks), min(lens[b], most) - 1, rope=rope, theta=500000.0,
                   slopes=slopes) for b in range(B)]
    check(o, lse, refs, "paged")


def test_no_lengths_and_scale():
    need_gpu()
    announce("paged without lengths")
    g = torch.Generator().manual_seed(1)
    k, v, table, flat = cache(2, 2, 96, 64, 32, g)
    q = torch.randn(2, 6, 64, generator=g).bfloat16().cuda()
    o, lse = api.attnfuse_decode_paged(q, k, v, table, scale=0.3, mask="none")
    check(o, lse, [decode(q[b], *flat[b], torch.arange(96), 95, scale=0.3) for b in range(2)], "all")


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -3e38])
@pytest.mark.parametrize("page,S,L,window,sinks", [(16, 500, 413, 0, 0), (64, 640, 555, 100, 5), (32, 3200, 3001, 70, 33),
                                                   (16, 160, 1, 0, 0)])
def test_what_is_not_visible_is_never_used(page, S, L, window, sinks, fill):
    """Everything that the query does not see holds NaN, infinities or the lowest values, free pages too."""
    need_gpu()
    announce(f"paged hidden page={page} S={S} L={L} W={window} sinks={sinks} fill={fill}")
    g = torch.Generator().manual_seed(S)
    k, v, table, flat = cache(1, 2, S, 128, page, g)
    q = torch.randn(1, 8, 128, generator=g).bfloat16().cuda()
    seen = seen_of(L, S, window, sinks)
    kept = torch.zeros(table.shape[1] * page, dtype=torch.bool)
    kept[seen] = True
    for x, y in ((k, flat[0][0]), (v, flat[0][1])):
        x.fill_(fill)
        x[table[0].long()] = torch.where(kept[None, :, None], y, torch.tensor(fill).bfloat16()).reshape(2, -1, page, 128) \
            .transpose(0, 1).cuda()
    table[0, -(-L // page):] = -7     # behind the length: any entries
    mask = dict(mask="sliding_window", window=window, sinks=sinks) if window else dict(mask="causal")
    o, lse = api.attnfuse_decode_paged(q, k, v, table, torch.tensor([L], dtype=torch.int32).cuda(), rope="neox", **mask)
    check(o, lse, [decode(q[0], *flat[0], seen, L - 1, rope="neox")], "hidden")
    if sinks:   # the same over a contiguous cache
        kc, vc = (torch.where(kept[None, :, None], y, torch.tensor(fill).bfloat16())[None].cuda() for y in flat[0])
        o, lse = api.attnfuse_decode(q, kc.contiguous(), vc.contiguous(), torch.tensor([L], dtype=torch.int32).cuda(),
                                     rope="neox", **mask)
        check(o, lse, [decode(q[0], *flat[0], seen, L - 1, rope="neox")], "hidden, contiguous")


def test_entries_outside_the_pool_hold_no_keys():
    need_gpu()
    announce("paged bad pages")
    g = torch.Generator().manual_seed(3)
    B, page, S = 3, 16, 480
    k, v, table, flat = cache(B, 2, S, 64, page, g)
    q = torch.randn(B, 4, 64, generator=g).bfloat16().cuda()
    gone = {0: [0, 3, 4, 29], 1: list(range(30)), 2: [17]}
    for b, entries in gone.items():
        for n, e in enumerate(entries):
            table[b, e] = (-1, k.shape[0], 2 ** 31 - 1, -2 ** 31)[n % 4]
    o, lse = api.attnfuse_decode_paged(q, k, v, table)
    at = torch.arange(S)
    refs = [decode(q[b], *flat[b], at[~torch.isin(at // page, torch.tensor(gone[b]))], S - 1) for b in range(B)]
    check(o, lse, refs, "bad pages")


def test_pages_that_sequences_share():
    """A page in several places of the table: a prefix two sequences share, and one page twice in a sequence; 20 and 5 heads
    a group."""
    need_gpu()
    announce("paged: shared pages")
    g = torch.Generator().manual_seed(9)
    page, D, most = 32, 128, 6
    table = torch.tensor([[3, 1, 4, 0, 0, 2], [3, 1, 4, 5, 1, 3]])
    lens = [180, 97]
    for H, Hkv in ((20, 1), (10, 2)):
        k, v = (torch.randn(7, Hkv, page, D, generator=g).bfloat16() for _ in "kv")
        q = torch.randn(2, H, D, generator=g).bfloat16()
        o, lse = api.attnfuse_decode_paged(q.cuda(), k.cuda(), v.cuda(), table.to(torch.int32).cuda(),
                                           torch.tensor(lens, dtype=torch.int32).cuda(), rope="neox")
        flat = [[x[table[b]].transpose(0, 1).reshape(Hkv, most * page, D) for x in (k, v)] for b in range(2)]
        check(o, lse, [decode(q[b], *flat[b], seen_of(lens[b], most * page, 0, 0), lens[b] - 1, rope="neox", theta=10000.0,
                              slopes=None) for b in range(2)], f"shared pages H={H}")


def test_a_sequence_does_not_depend_on_the_others():
    need_gpu()
    announce("paged neighbours")
    g = torch.Generator().manual_seed(4)
    B, S = 20, 3000
    k, v, table, _ = cache(B, 4, S, 128, 32, g)
    q = torch.randn(B, 16, 128, generator=g).bfloat16().cuda()
    nbytes = api.attnfuse_decode_paged_workspace_bytes(B, 16, 4, table.shape[1] * 32, 128)

    def run(lens, fill):
        ws = torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")
        return api.attnfuse_decode_paged(q, k, v, table, torch.tensor(lens, dtype=torch.int32).cuda(), rope="neox", workspace=ws)

    want = run([2005] + [S] * (B - 1), 0)
    for others in ([0] * (B - 1), [(37 * b) % S for b in range(1, B)]):
        got = run([2005] + others, 0xFF)
        assert torch.equal(got[0][0], want[0][0]) and torch.equal(got[1][0], want[1][0])
    with_lens, without = run([table.shape[1] * 32] * B, 0), api.attnfuse_decode_paged(q, k, v, table, rope="neox")
    assert all(torch.equal(a, b) for a, b in zip(with_lens, without))


@pytest.mark.parametrize("B,H,Hkv,S,D,lens,window,sinks,rope", [
    (1, 8, 2, 33, 64, [33], 4, 2, "neox"), (3, 32, 8, 1001, 128, [1001, 500, 3], 128, 4, "none"),
    (2, 12, 12, 2047, 64, None, 300, 77, "interleaved"), (4, 8, 1, 513, 128, [0, 513, 600, 257], 64, 64, "neox"),
    (1, 4, 4, 100000, 128, [99999], 4096, 4, "neox")], ids=lambda x: str(x)[:18])
def test_contiguous_with_sinks(B, H, Hkv, S, D, lens, window, sinks, rope):
    need_gpu()
    announce(f"stream B={B} H={H}/{Hkv} S={S} D={D} W={window} sinks={sinks} {rope}")
    g = torch.Generator().manual_seed(S)
    q = torch.randn(B, H, D, generator=g).bfloat16()
    k, v = (torch.randn(B, Hkv, S, D, generator=g).bfloat16() for _ in "kv")
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
    o, lse = api.attnfuse_decode(q.cuda(), k.cuda(), v.cuda(), ln, rope=rope, theta=500000.0, mask="sliding_window",
                                 window=window, sinks=sinks)
    lens = lens or [S] * B
    refs = [decode(q[b], k[b], v[b], seen_of(lens[b], S, window, sinks), min(lens[b], S) - 1, rope=rope, theta=500000.0)
            for b in range(B)]
    check(o, lse, refs, "stream")


def test_offsets_past_32_bits():
    """Pages that lie past 2^32 bytes of their pool (as a slice of a larger one), the last page of the pool among them."""
    need_gpu()
    announce("paged far pages")
    g = torch.Generator().manual_seed(5)
    pages, page, D = 48, 16, 128
    pool = torch.empty(pages, 56 << 20, dtype=torch.bfloat16, device="cuda")   # 112 MiB apart: 5.25 GiB
    k = pool.as_strided((pages, 2, page, D), (56 << 20, page * D, D, 1))
    v = pool.as_strided((pages, 2, page, D), (56 << 20, page * D, D, 1), 1 << 20)
    flat = [torch.randn(pages, 2, page, D, generator=g).bfloat16() for _ in "kv"]
    k.copy_(flat[0])
    v.copy_(flat[1])
    order = torch.arange(pages - 1, -1, -1)
    q = torch.randn(1, 4, D, generator=g).bfloat16().cuda()
    o, lse = api.attnfuse_decode_paged(q, k, v, order.to(torch.int32)[None].cuda(), rope="neox")
    keys, values = (x[order].transpose(0, 1).reshape(2, -1, D) for x in flat)
    check(o, lse, [decode(q[0], keys, values, torch.arange(pages * page), pages * page - 1, rope="neox")], "far")


def test_replayed_from_a_graph():
    """A serving step, append then decode, captured once and replayed as the sequences grow, against eager calls."""
    need_gpu()
    announce("paged graph")
    g = torch.Generator().manual_seed(6)
    B, H, Hkv, D, page, n = 3, 8, 2, 128, 16, 12
    lens = torch.tensor([5, 100, 31], dtype=torch.int32).cuda()
    table = torch.randperm(B * n, generator=g).to(torch.int32).reshape(B, n).cuda()
    pools = [torch.randn(B * n, Hkv, page, D, generator=g).bfloat16().cuda() for _ in "kv"]
    pools += [x.clone() for x in pools]
    w = (1 + 0.1 * torch.randn(D, generator=g)).bfloat16().cuda()
    x = torch.empty(B, H + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    rows = torch.arange(B).cuda()

    def step(x, lens, k, v):
        pos = lens - 1
        slots = table[rows, (pos // page).long()].long() * page + pos % page
        q = api.attnfuse_qknorm_rope_append(x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], k, v, slots, w, w, theta=500000.0,
                                            positions=pos, max_positions=4096)
        return (q,) + tuple(api.attnfuse_decode_paged(q, k, v, table, lens, mask="sliding_window", window=40, sinks=4))

    x.normal_(generator=torch.Generator("cuda").manual_seed(1))
    step(x, lens, *pools[:2])   # builds the table
    pools[0].copy_(pools[2])
    pools[1].copy_(pools[3])
    static = lens.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step(x, static, *pools[:2])
    for i in range(4):
        x.normal_(generator=torch.Generator("cuda").manual_seed(10 + i))
        static.copy_(lens + i)
        graph.replay()
        torch.cuda.synchronize()
        want = step(x, lens + i, *pools[2:])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])


def test_on_two_streams():
    need_gpu()
    announce("paged streams")
    g = torch.Generator().manual_seed(7)
    sets = [cache(4, 2, 4000, 128, 16, g)[:3] for _ in range(2)]
    qs = [torch.randn(4, 8, 128, generator=g).bfloat16().cuda() for _ in range(2)]
    want = [api.attnfuse_decode_paged(q, *s, rope="neox") for q, s in zip(qs, sets)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = api.attnfuse_decode_paged(qs[i], *sets[i], rope="neox")
    torch.cuda.synchronize()
    assert all(torch.equal(got[i][j], want[i][j]) for i in range(2) for j in range(2))


def test_the_longest_first():
    """More workgroups than are resident, each with a long share: the sequences are taken by length.  Equal, empty, negative
    and over-long ones among them; each result is that of the sequence alone."""
    need_gpu()
    announce("paged by length")
    g = torch.Generator().manual_seed(11)
    B, H, Hkv, S, D, page = 37, 32, 16, 1100, 128, 16
    lens = torch.randint(1, S + 1, (B,), generator=g).to(torch.int32)
    lens[3], lens[4], lens[5], lens[6], lens[20], lens[21], lens[36] = 0, -5, 5000, 700, 700, 700, 1
    k, v, table, flat = cache(B, Hkv, S, D, page, g)
    q = torch.randn(B, H, D, generator=g).bfloat16().cuda()
    most = table.shape[1] * page
    o, lse = api.attnfuse_decode_paged(q, k, v, table, lens.cuda(), rope="neox")
    for b in range(B):
        want = decode(q[b], *flat[b], seen_of(int(lens[b]), most, 0, 0), min(int(lens[b]), most) - 1, rope="neox")
        check(o[b:b + 1], lse[b:b + 1], [want], f"sequence {b}")


# ---------------------------------------------------------------- NaN among what is visible
def shares(nbytes, B, H, D):
    """Workgroups that share a sequence, from the workspace: a (max, sum) and D values for each, rounded up."""
    return nbytes // (B * H * (4 * D + 8))


def check_nan(o, lse, ref, nan_heads, what):
    """O and LSE of one sequence: NaN in every element of the given heads, the reference's values in the others."""
    O, L, pv, mag = ref
    bad = torch.zeros(o.shape[0], dtype=torch.bool)
    bad[nan_heads] = True
    assert torch.equal(o.cpu().isnan(), bad[:, None].expand(*o.shape)), f"{what}: O's NaN"
    assert torch.equal(lse.cpu().isnan(), bad), f"{what}: LSE's NaN"
    check(o[~bad.to(o.device)][None], lse[~bad.to(o.device)][None], [(O[~bad], L[~bad], pv[~bad], mag[~bad])], what)


@pytest.mark.parametrize("rope", ["none", "neox"])
@pytest.mark.parametrize("H,Hkv,D,S,L,split", [(8, 2, 128, 100, 97, 1), (8, 2, 64, 2048, 641, 16), (4, 1, 128, 4096, 4096, 32),
                                               (6, 3, 64, 4096, 129, 32)])
def test_a_nan_query_or_key_gives_nan(H, Hkv, D, S, L, split, rope):
    """NaN scores come out as NaN whether one workgroup takes the sequence or several, which are joined, and never as the
    result of a sequence without visible keys, which stays O = 0 and LSE = -inf beside them."""
    need_gpu()
    announce(f"paged NaN H={H}/{Hkv} D={D} S={S} L={L} {rope}")
    g = torch.Generator().manual_seed(S + L)
    G, page = H // Hkv, 16
    k, v, table, flat = cache(1, Hkv, S, D, page, g)
    nbytes = api.attnfuse_decode_paged_workspace_bytes(1, H, Hkv, table.shape[1] * page, D)
    assert shares(nbytes, 1, H, D) == split
    q = torch.randn(1, H, D, generator=g).bfloat16()
    lens = torch.tensor([L], dtype=torch.int32).cuda()
    ref = decode(q[0], *flat[0], torch.arange(L), L - 1, rope=rope)
    bad = q.clone()
    bad[0, 1] = float("nan")
    o, lse = api.attnfuse_decode_paged(bad.cuda(), k, v, table, lens, rope=rope)
    check_nan(o[0], lse[0], ref, [1], "a NaN query")
    # one visible key, the last (alone in its tile where L is 32 n + 1), and every key, of the last K/V head
    for n, what in ((slice(L - 1, L), "the last key NaN"), (slice(0, L), "every key NaN")):
        kn = k.clone()
        for i in range(*n.indices(L)):
            kn[table[0, i // page].long(), Hkv - 1, i % page] = float("nan")
        o, lse = api.attnfuse_decode_paged(q.cuda(), kn, v, table, lens, rope=rope)
        check_nan(o[0], lse[0], ref, list(range(H - G, H)), what)
    for pages, n in ((table, torch.zeros_like(lens)), (torch.full_like(table, -1), lens)):
        o, lse = api.attnfuse_decode_paged(bad.cuda(), k, v, pages, n, rope=rope)
        assert not o.any() and torch.isneginf(lse).all(), "no visible key"


@pytest.mark.parametrize("S,L,window,sinks,split", [(70, 70, 40, 4, 1), (6000, 5001, 4096, 4, 32)])
def test_a_nan_query_or_key_gives_nan_in_a_contiguous_cache(S, L, window, sinks, split):
    need_gpu()
    announce(f"stream NaN S={S} L={L} W={window} sinks={sinks}")
    g = torch.Generator().manual_seed(S)
    H, Hkv, D = 8, 2, 128
    nbytes = api.attnfuse_decode_paged_workspace_bytes(2, H, Hkv, S, D, window, sinks)
    assert shares(nbytes, 2, H, D) == split
    q = torch.randn(2, H, D, generator=g).bfloat16()
    k, v = (torch.randn(2, Hkv, S, D, generator=g).bfloat16() for _ in "kv")
    lens = torch.tensor([L, 0], dtype=torch.int32).cuda()
    ref = decode(q[0], k[0], v[0], seen_of(L, S, window, sinks), L - 1, rope="neox")
    bad, kn = q.clone(), k.clone()
    bad[:, 3] = float("nan")
    kn[0, 0, 1] = float("nan")   # a sink
    for a, b, heads in ((bad, k, [3]), (q, kn, [0, 1, 2, 3])):
        o, lse = api.attnfuse_decode(a.cuda(), b.cuda(), v.cuda(), lens, rope="neox", mask="sliding_window", window=window,
                                     sinks=sinks)
        check_nan(o[0], lse[0], ref, heads, "stream")
        assert not o[1].any() and torch.isneginf(lse[1]).all()


@pytest.mark.parametrize("S", [100, 4096])
def test_a_nan_value_gives_nan_in_its_element(S):
    need_gpu()
    announce(f"paged NaN value S={S}")
    g = torch.Generator().manual_seed(S)
    k, v, table, flat = cache(1, 2, S, 64, 16, g)
    q = torch.randn(1, 4, 64, generator=g).bfloat16()
    o, lse = api.attnfuse_decode_paged(q.cuda(), k, v, table)
    v[table[0, 3].long(), 1, 5, 33] = float("nan")
    on, ln = api.attnfuse_decode_paged(q.cuda(), k, v, table)
    assert torch.equal(ln, lse) and on[0, 2:, 33].isnan().all()
    on[0, 2:, 33] = o[0, 2:, 33]
    assert torch.equal(on, o)
