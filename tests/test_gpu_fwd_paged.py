"""New tokens over a paged cache, behind a prefix that the batch shares (attnfuse_fwd_paged, and decode_paged with a prefix),
against the definition in 64 bits.  Tolerances: paged_ref.check."""
import pytest
import torch

from gpu_util import announce, need_gpu
from llm_ref import f64
from paged_ref import batch, check
from paper_2609_13612_amd import api

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def pool(n, Hkv, page, D, g, nhd=False):
    shape = (n, page, Hkv, D) if nhd else (n, Hkv, page, D)
    k, v = (torch.randn(shape, generator=g).bfloat16().cuda() for _ in "kv")
    return (k.transpose(1, 2), v.transpose(1, 2)) if nhd else (k, v)


def setup(counts, lens, H, Hkv, D, page, P, g, nhd=False, pad=0, front=0, wide=0):
    """Queries, pages in a random order, tables and starts (front: tokens before the first sequence; pad: behind the last;
    wide: pages more than the longest sequence has)."""
    B, most, ahead = len(counts), max(1, -(-max(max(lens), 1) // page)) + wide, -(-P // page)
    k, v = pool(B * most + ahead + 2, Hkv, page, D, g, nhd)
    order = torch.randperm(B * most + ahead + 2, generator=g).to(torch.int32)
    starts = [front]
    for n in counts:
        starts.append(starts[-1] + n)
    q = torch.randn(starts[-1] + pad, H, D, generator=g).bfloat16().cuda()
    return q, k, v, order[:B * most].reshape(B, most).cuda(), starts, order[B * most:B * most + ahead].cuda() if P else None


CASES = [
    # tokens, own keys, H, Hkv, D, page, prefix, places first, padding, front
    ([1], [1], 2, 1, 64, 16, 0, False, 0, 0),
    ([5], [5], 8, 2, 128, 16, 0, False, 0, 0),
    ([64, 64], [64, 200], 4, 2, 64, 64, 0, False, 3, 0),
    ([130, 1, 17, 33], [130, 1000, 17, 600], 8, 2, 128, 16, 0, True, 0, 0),
    ([3, 0, 7], [50, 20, 0], 6, 2, 64, 32, 0, False, 5, 4),            # nobody's tokens, no queries, more queries than keys
    ([40, 2], [30, 1], 5, 5, 128, 16, 100, False, 0, 0),               # the same behind a prefix
    ([12, 30, 1, 5], [12, 40, 77, 500], 32, 8, 128, 16, 1000, False, 9, 2),
    ([25, 60], [25, 90], 12, 12, 64, 128, 4001, True, 0, 0),
    ([300, 257], [300, 900], 16, 2, 128, 64, 777, False, 0, 0),        # rows enough to walk both
    ([1000], [1500], 8, 1, 64, 16, 333, False, 10, 0),
    ([9] * 70, [9 + i for i in range(70)], 3, 1, 64, 16, 65, False, 0, 0),
    ([2, 3], [2, 3], 40, 1, 128, 1024, 64, False, 0, 0),               # long pages, 40 heads a group
    ([200], [200], 48, 3, 128, 16, 63, True, 0, 7),
    ([700, 1, 1], [6000, 1, 64], 4, 4, 64, 16, 0, False, 0, 0),
]


@pytest.mark.parametrize("counts,lens,H,Hkv,D,page,P,nhd,pad,front", CASES, ids=lambda x: str(x)[:20].replace(" ", ""))
def test_prompts(counts, lens, H, Hkv, D, page, P, nhd, pad, front):
    need_gpu()
    announce(f"fwd_paged tokens={counts[:5]} keys={lens[:5]} H={H}/{Hkv} D={D} page={page} P={P} nhd={nhd} pad={pad} front={front}")
    g = torch.Generator().manual_seed(sum(counts) + P)
    q, k, v, table, starts, prefix = setup(counts, lens, H, Hkv, D, page, P, g, nhd, pad, front, wide=1)
    T, B = q.shape[0], len(counts)
    out, lse = torch.full_like(q, 7.0), torch.full((T, H), 7.0, device="cuda")
    nbytes = api.attnfuse_fwd_paged_workspace_bytes(T, B, H, Hkv, D, table.shape[1] * page, 0 if prefix is None else len(prefix) * page)
    guard = torch.full((nbytes + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    kw = dict(prefix_table=prefix, prefix_len=i32([P]) if P else None)
    o, l = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), out=out, lse=lse, workspace=guard[:nbytes], **kw)
    torch.cuda.synchronize()
    assert o is out and l is lse
    assert (guard[nbytes:] == 0x5A).all(), "written past the workspace"
    check(o, l, batch(q, k, v, table, starts, lens, prefix, P), "prompts")
    for rows in (slice(0, front), slice(starts[-1], T)):
        assert (o[rows] == 7).all() and (l[rows] == 7).all(), "rows of no sequence"
    again = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), **kw)
    some = slice(front, starts[-1])
    assert torch.equal(again[0][some], o[some]) and torch.equal(again[1][some], l[some]), "another call, other bits"


DECODE = [
    # own keys, H, Hkv, D, page, prefix
    ([1], 2, 1, 64, 16, 1),
    ([0, 5, 0], 8, 2, 128, 16, 0),                        # a prefix of no keys in one page: empty rows
    ([60, 1, 0, 17], 32, 8, 128, 16, 500),
    ([700, 33, 1000], 12, 12, 64, 32, 2049),
    ([(13 * i) % 300 for i in range(90)], 16, 4, 128, 64, 4000),
    ([5, 6], 40, 1, 64, 16, 130),
    ([3, 400], 300, 1, 64, 16, 64),                       # more heads a group than a tile has rows
]


@pytest.mark.parametrize("lens,H,Hkv,D,page,P", DECODE, ids=lambda x: str(x)[:20].replace(" ", ""))
def test_decode(lens, H, Hkv, D, page, P):
    need_gpu()
    announce(f"decode behind a prefix keys={lens[:5]} H={H}/{Hkv} D={D} page={page} P={P}")
    g = torch.Generator().manual_seed(len(lens) + P)
    B = len(lens)
    q, k, v, table, starts, prefix = setup([1] * B, lens, H, Hkv, D, page, max(P, 1), g)
    o, lse = api.attnfuse_decode_paged(q, k, v, table, i32(lens), prefix_table=prefix, prefix_len=i32([P]))
    refs = batch(q, k, v, table, starts, lens, prefix, P)
    check(o, lse, refs, "decode")
    o2, lse2 = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), prefix_table=prefix, prefix_len=i32([P]))
    check(o2, lse2, refs, "decode as prompts")


def test_whole_pages_without_lengths_and_a_scale():
    need_gpu()
    announce("fwd_paged without lengths")
    g = torch.Generator().manual_seed(1)
    q, k, v, table, starts, prefix = setup([3, 30], [96, 96], 6, 2, 64, 32, 64, g)
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), prefix_table=prefix, scale=0.3)
    check(o, lse, batch(q, k, v, table, starts, [96, 96], prefix, 64, scale=0.3), "all")
    # lengths beyond what the tables hold are clamped, negative ones are 0
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32([9999, -4]), prefix_table=prefix, prefix_len=i32([9999]))
    check(o, lse, batch(q, k, v, table, starts, [96, 0], prefix, 64), "clamped")
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32([96, 96]), prefix_table=prefix, prefix_len=i32([-1]))
    check(o, lse, batch(q, k, v, table, starts, [96, 96], prefix, 0), "no prefix")


def test_agrees_with_decode_over_pages():
    """One token each and no prefix is decode over pages (queries already rotated)."""
    need_gpu()
    announce("fwd_paged as decode_paged")
    g = torch.Generator().manual_seed(2)
    lens = [400, 1, 37, 129]
    q, k, v, table, starts, _ = setup([1] * 4, lens, 8, 2, 128, 16, 0, g)
    refs = batch(q, k, v, table, starts, lens)
    check(*api.attnfuse_decode_paged(q, k, v, table, i32(lens)), refs, "decode")
    check(*api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens)), refs, "prompts")


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -3e38])
@pytest.mark.parametrize("counts,lens,P,page", [([1, 1], [1, 70], 33, 16), ([20, 7], [20, 90], 100, 64), ([300], [333], 65, 16),
                                                ([40], [400], 0, 32)])
def test_what_is_no_key_is_never_used(counts, lens, P, page, fill):
    """Pages of nobody, places behind the lengths and behind the prefix's end hold NaN, infinities or the lowest values."""
    need_gpu()
    announce(f"fwd_paged hidden {counts} {lens} P={P} page={page} {fill}")
    g = torch.Generator().manual_seed(3)
    q, k, v, table, starts, prefix = setup(counts, lens, 8, 2, 128, page, P, g, wide=2)
    kept = torch.zeros(k.shape[0], page, dtype=torch.bool)
    for pages, n in [(table[b].cpu(), lens[b]) for b in range(len(lens))] + ([(prefix.cpu(), P)] if P else []):
        at = torch.arange(n)
        kept[pages.long()[at // page], at % page] = True
    for x in (k, v):
        x.copy_(torch.where(kept[:, None, :, None], x.cpu(), torch.tensor(fill).bfloat16()).cuda())
    for b, n in enumerate(lens):
        table[b, -(-n // page):] = -7   # behind the length: any entries
    kw = dict(prefix_table=prefix, prefix_len=i32([P])) if P else {}
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), **kw)
    check(o, lse, batch(q, k, v, table, starts, lens, prefix, P), "hidden")


def test_entries_outside_the_pool_hold_no_keys():
    need_gpu()
    announce("fwd_paged bad pages")
    g = torch.Generator().manual_seed(4)
    lens, counts, P, page = [100, 64, 40], [30, 1, 40], 200, 16
    q, k, v, table, starts, prefix = setup(counts, lens, 8, 4, 64, page, P, g)
    bad = [-1, k.shape[0], 2 ** 31 - 1, -2 ** 31]
    table[0, 1], table[0, 3], table[1, 0], table[2, 2] = bad
    prefix[0], prefix[5], prefix[12] = bad[1], bad[0], bad[3]
    kw = dict(prefix_table=prefix, prefix_len=i32([P]))
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), **kw)
    check(o, lse, batch(q, k, v, table, starts, lens, prefix, P), "bad pages")
    table.fill_(-1)
    prefix.fill_(k.shape[0])   # nothing at all: empty rows
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), **kw)
    assert not o.any() and torch.isneginf(lse).all()


def test_starts_outside_the_tokens_are_clamped():
    need_gpu()
    announce("fwd_paged starts")
    g = torch.Generator().manual_seed(5)
    q, k, v, table, _, _ = setup([10, 10], [64, 64], 4, 2, 64, 16, 0, g)
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32([-5, 8, 900]), i32([64, 64]))
    check(o, lse, batch(q, k, v, table, [0, 8, 20], [64, 64]), "clamped")


@pytest.mark.parametrize("count", [1, 40, 300])
def test_nan_stays_nan(count):
    """A NaN in a query makes its row NaN and no other; one in a key of the prefix, every row."""
    need_gpu()
    announce(f"fwd_paged NaN {count}")
    g = torch.Generator().manual_seed(6)
    q, k, v, table, starts, prefix = setup([count, count], [count + 9] * 2, 4, 2, 64, 16, 700, g)
    kw = dict(prefix_table=prefix, prefix_len=i32([700]))
    lens = i32([count + 9] * 2)
    want = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), lens, **kw)
    q[count, 1, 3] = float("nan")
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), lens, **kw)
    hit = torch.zeros(2 * count, 4, dtype=torch.bool, device="cuda")
    hit[count, 1] = True
    assert o[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(o[~hit], want[0][~hit]) and torch.equal(lse[~hit], want[1][~hit])
    k[prefix[20].long(), 0, 5, 9] = float("nan")
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), lens, **kw)
    assert o[:, :2].isnan().all() and lse[:, :2].isnan().all() and o[:, 2:].isfinite().all()


def test_large_scores():
    """Scores of thousands, one key to a row: the maxima of partials lie far apart."""
    need_gpu()
    announce("fwd_paged large scores")
    g = torch.Generator().manual_seed(7)
    q, k, v, table, starts, prefix = setup([6, 1], [300, 20], 8, 2, 128, 16, 5000, g)
    q *= 30
    k *= 30
    kw = dict(prefix_table=prefix, prefix_len=i32([5000]))
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32([300, 20]), **kw)
    check(o, lse, batch(q, k, v, table, starts, [300, 20], prefix, 5000), "large")


def test_native_and_python_marshalling_agree(monkeypatch):
    need_gpu()
    announce("fwd_paged marshalling")
    assert api._native is not None, "the native binding is not built"
    g = torch.Generator().manual_seed(8)
    q, k, v, table, starts, prefix = setup([1, 1, 1], [30, 40, 2], 8, 4, 64, 16, 90, g, nhd=True)
    kw = dict(prefix_table=prefix, prefix_len=i32([88]))
    taken, real = [], api._native

    class Spy:
        def __getattr__(self, name):
            def call(*args):
                r = getattr(real, name)(*args)
                taken.append((name, r is not None))
                return r
            return call

    def calls():
        return (*api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32([30, 40, 2]), **kw),
                *api.attnfuse_decode_paged(q, k, v, table, i32([30, 40, 2]), **kw),
                *api.attnfuse_fwd_paged(q, k, v, table, i32(starts), scale=0.2))

    monkeypatch.setattr(api, "_native", Spy())
    a = calls()
    assert taken == [("fwd_paged", True)] * 3
    monkeypatch.setattr(api, "_native", None)
    assert all(torch.equal(x, y) for x, y in zip(a, calls()))


@pytest.mark.parametrize("native", [True, False])
def test_refusals(monkeypatch, native):
    need_gpu()
    announce(f"fwd_paged refusals native={native}")
    if not native:
        monkeypatch.setattr(api, "_native", None)
    g = torch.Generator().manual_seed(9)
    q, k, v, table, starts, prefix = setup([2, 2], [30, 40], 8, 4, 64, 16, 90, g)
    s, lens, plen = i32(starts), i32([30, 40]), i32([90])
    for bad in (dict(starts=s[:2]), dict(starts=s.long()), dict(starts=None), dict(lens=lens[:1]), dict(lens=lens.cpu()),
                dict(table=table.long()), dict(table=table[0]), dict(q=q.float()), dict(q=q[:, :, :32]), dict(v=v[:, :, :8]),
                dict(prefix=prefix.long()), dict(prefix=prefix[None]), dict(plen=plen.expand(2).contiguous()),
                dict(prefix=None), dict(prefix=prefix[:0]), dict(out=torch.empty_like(q[:1])), dict(lse=torch.empty(4, 8))):
        a = dict(q=q, k=k, v=v, table=table, starts=s, lens=lens, prefix=prefix, plen=plen, out=None, lse=None)
        a.update(bad)
        with pytest.raises((ValueError, TypeError)):
            api.attnfuse_fwd_paged(a["q"], a["k"], a["v"], a["table"], a["starts"], a["lens"], prefix_table=a["prefix"],
                                   prefix_len=a["plen"], out=a["out"], lse=a["lse"])
    one = dict(prefix_table=prefix, prefix_len=plen)
    for bad in (dict(rope="neox"), dict(mask="sliding_window", window=4), dict(alibi_slopes=torch.ones(8, device="cuda")),
                dict(mask="sliding_window", window=4, sinks=1)):
        with pytest.raises(ValueError):
            api.attnfuse_decode_paged(q[:2], k, v, table, lens, **one, **bad)
    with pytest.raises(ValueError):
        api.attnfuse_decode_paged(q, k, v, table, lens, **one)   # four queries, two sequences
    with pytest.raises(api.AttnFuseError):
        api.attnfuse_fwd_paged(q, k, v, table, s, lens, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"), **one)


def test_two_graphs_share_a_workspace():
    """Captured decode and prompt calls, one after the other through one workspace, replayed with the program's own work
    between them."""
    need_gpu()
    announce("fwd_paged graphs")
    g = torch.Generator().manual_seed(10)
    q, k, v, table, starts, prefix = setup([40, 3, 1], [50, 60, 64], 8, 2, 128, 16, 900, g, wide=1)
    s, lens, plen = i32(starts), i32([50, 60, 64]), i32([900])
    one = torch.randn(3, 8, 128, generator=g).bfloat16().cuda()
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    kw = dict(prefix_table=prefix, prefix_len=plen, workspace=ws)
    graphs, outs = [], []
    for call in (lambda: api.attnfuse_fwd_paged(q, k, v, table, s, lens, **kw),
                 lambda: api.attnfuse_decode_paged(one, k, v, table, lens, **kw)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call())
        graphs.append(graph)
    for i in range(3):
        for t in (q, one, k, v):
            t.copy_(torch.randn(t.shape, generator=g).bfloat16().cuda())
        lens.copy_(i32([50 - i, 60 + i, 64]))
        plen.fill_(900 - 100 * i)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        other = dict(prefix_table=prefix, prefix_len=plen)
        want = (api.attnfuse_fwd_paged(q, k, v, table, s, lens, **other), api.attnfuse_decode_paged(one, k, v, table, lens, **other))
        assert all(torch.equal(a, b) for x, y in zip(outs, want) for a, b in zip(x, y)), f"replay {i}"


def test_two_streams_at_once():
    need_gpu()
    announce("fwd_paged streams")
    g = torch.Generator().manual_seed(11)
    jobs = [setup([200, 30], [300, 900], 16, 4, 128, 16, 3000, g), setup([1] * 16, [100] * 16, 16, 4, 128, 16, 6000, g)]
    call = lambda j: api.attnfuse_fwd_paged(j[0], j[1], j[2], j[3], i32(j[4]), prefix_table=j[5])   # noqa: E731
    want = [call(j) for j in jobs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in jobs], []
    for j, st in zip(jobs, streams):
        with torch.cuda.stream(st):
            got.append(call(j))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_offsets_past_32_bits():
    """Pages whose offsets in elements pass 2^32."""
    need_gpu()
    announce("fwd_paged far pages")
    g = torch.Generator().manual_seed(12)
    pages, Hkv, page, D = 20000, 8, 256, 128
    k = torch.zeros(pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert (pages - 1) * Hkv * page * D > 2 ** 32
    lens, counts, P = [300, 500], [3, 40], 600
    used = torch.tensor([19999, 2, 19990, 16400, 17000, 1, 18500], dtype=torch.int32)
    for x in (k, v):
        x[used.long().cuda()] = torch.randn(len(used), Hkv, page, D, generator=g).bfloat16().cuda()
    table, prefix = used[:4].reshape(2, 2).cuda(), used[4:].cuda()
    q = torch.randn(43, 16, D, generator=g).bfloat16().cuda()
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32([0, 3, 43]), i32(lens), prefix_table=prefix, prefix_len=i32([P]))
    order = {int(p): i for i, p in enumerate(used)}   # the same pages of a small pool
    small = [torch.tensor([[order[int(p)] for p in row] for row in x.reshape(-1, x.shape[-1])], dtype=torch.int32)
             for x in (table.cpu(), prefix.cpu())]
    ks, vs = k[used.long().cuda()], v[used.long().cuda()]
    check(o, lse, batch(q, ks, vs, small[0], [0, 3, 43], lens, small[1][0], P), "far")


def test_pages_named_twice():
    """A page may be in a table twice, in several sequences' and in the prefix's."""
    need_gpu()
    announce("fwd_paged shared pages")
    g = torch.Generator().manual_seed(15)
    q, k, v, table, starts, prefix = setup([20, 1, 5], [60, 64, 33], 8, 2, 64, 16, 200, g)
    prefix[7] = prefix[2]
    table[1] = table[0]
    table[2, 0], table[2, 1] = prefix[0], prefix[0]
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32([60, 64, 33]), prefix_table=prefix, prefix_len=i32([199]))
    check(o, lse, batch(q, k, v, table, starts, [60, 64, 33], prefix, 199), "shared pages")


@pytest.mark.parametrize("ahead", [True, False])
def test_longest_lists(ahead):
    """2^20 keys of a prefix, or of a sequence."""
    need_gpu()
    announce(f"fwd_paged 2^20 keys ahead={ahead}")
    g = torch.Generator().manual_seed(16)
    n, page = 1 << 20, 256
    q, k, v, table, starts, prefix = setup([3, 1], [n, 7] if not ahead else [10, 7], 2, 1, 64, page, n if ahead else 0, g)
    lens = [n, 7] if not ahead else [10, 7]
    kw = dict(prefix_table=prefix, prefix_len=i32([n])) if ahead else {}
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), **kw)
    check(o, lse, batch(q, k, v, table, starts, lens, prefix, n if ahead else 0), "2^20 keys")
    if ahead:
        with pytest.raises(api.AttnFuseError):
            api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), prefix_table=torch.cat((prefix, prefix[:1])))


def test_many_tokens():
    """Tokens by the ten thousands, of many sequences of any length: sampled against the definition."""
    need_gpu()
    announce("fwd_paged many tokens")
    g = torch.Generator().manual_seed(17)
    counts = [int(x) for x in torch.randint(0, 90, (700,), generator=g)]
    lens = [c + int(x) for c, x in zip(counts, torch.randint(0, 60, (700,), generator=g))]
    q, k, v, table, starts, prefix = setup(counts, lens, 4, 2, 64, 16, 90, g, pad=5)
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), prefix_table=prefix, prefix_len=i32([90]))
    pick = [0, 1, 63, 64, 65, 127, 128, 350, 640, 698, 699]
    kc, vc = k.cpu(), v.cpu()
    for b in pick:
        at = [starts[b], starts[b + 1]]
        refs = batch(q, kc, vc, table[b:b + 1], at, [lens[b]], prefix, 90)
        check(o, lse, refs, f"sequence {b}")


@pytest.mark.parametrize("P", [0, 100])
@pytest.mark.parametrize("B", [2, 40, 64])
def test_longest_first(B, P):
    """More workgroups than run at once, of up to 64 sequences: they go by length, with ties, empty ones and lengths beyond
    the table among them.  The lengths alone decide, whatever rows there are."""
    need_gpu()
    announce(f"fwd_paged longest first B={B} P={P}")
    g = torch.Generator().manual_seed(19 + B)
    H = 64 if B > 2 else 400
    counts = [int(x) for x in torch.randint(0, 30, (B,), generator=g)]
    counts[0] = 140
    lens = [c + int(x) for c, x in zip(counts, torch.randint(0, 200, (B,), generator=g))]
    lens[1] = lens[0] = 300
    if B > 2:
        lens[5], lens[7], counts[9] = 0, -3, 0
    q, k, v, table, starts, prefix = setup(counts, lens, H, H, 64, 16, P, g, pad=3)
    lens[-1] = 9999
    kw = dict(prefix_table=prefix, prefix_len=i32([P])) if P else {}
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), **kw)
    few = slice(0, 3)   # heads: the reference of three of them
    refs = batch(q[:, few], k[:, few], v[:, few], table, starts, lens, prefix, P)
    check(o[:, few], lse[:, few], refs, "prompts")
    last = slice(H - 2, H)
    check(o[:, last], lse[:, last], batch(q[:, last], k[:, last], v[:, last], table, starts, lens, prefix, P), "prompts, last heads")
    if P:
        o, lse = api.attnfuse_decode_paged(q[:B].contiguous(), k, v, table, i32(lens), **kw)
        refs = batch(q[:B, few], k[:, few], v[:, few], table, list(range(B + 1)), lens, prefix, P)
        check(o[:, few], lse[:, few], refs, "decode")


ONE = [
    # own keys, H, Hkv, D, page, prefix
    ([(37 * i) % 3000 for i in range(40)], 16, 16, 64, 16, 100),   # lists of 47 tiles, and none
    ([5, 70], 2, 1, 64, 256, 131077),                              # a prefix's shares of 32 tiles
    ([7], 32, 1, 128, 16, 5000),                                   # 32 rows behind the prefix
    ([7, 9], 17, 1, 64, 16, 5000),                                 # 34 there, 17 of their own
    ([33, 2000, 0], 64, 2, 128, 16, 40),                           # 32 heads a group
    ([33, 2000, 0], 66, 2, 128, 16, 40),                           # 33
    ([33, 2000, 0], 64, 2, 128, 32, 0),                            # no prefix
    ([64 - i % 9 for i in range(130)], 8, 8, 128, 16, 0),          # one share of each list: nothing to join
    ([31, 32, 33, 63, 64, 65, 1], 3, 1, 64, 16, 0),
    ([95, 96, 97, 127, 128, 129, 130], 4, 4, 128, 64, 33),
]


@pytest.mark.parametrize("lens,H,Hkv,D,page,P", ONE, ids=lambda x: str(x)[:20].replace(" ", ""))
def test_one_token_each(lens, H, Hkv, D, page, P):
    """Up to 32 rows a list, and just more.  Places that hold no key are NaN; entries behind the lengths, and one in the middle
    of a long list, name no page."""
    need_gpu()
    announce(f"one token each keys={lens[:5]} B={len(lens)} H={H}/{Hkv} D={D} page={page} P={P}")
    g = torch.Generator().manual_seed(21 + len(lens) + P)
    B = len(lens)
    q, k, v, table, starts, prefix = setup([1] * B, lens, H, Hkv, D, page, P, g, wide=1)
    kept = torch.zeros(k.shape[0], page, dtype=torch.bool)
    for pages, n in [(table[b].cpu(), lens[b]) for b in range(B)] + ([(prefix.cpu(), P)] if P else []):
        at = torch.arange(n)
        kept[pages.long()[at // page], at % page] = True
    for x in (k, v):
        x.copy_(torch.where(kept[:, None, :, None], x.cpu(), torch.tensor(float("nan")).bfloat16()).cuda())
    for b, n in enumerate(lens):
        used = -(-n // page)
        table[b, used:] = -7
        if used > 2:
            table[b, used // 2] = k.shape[0]
    nbytes = api.attnfuse_fwd_paged_workspace_bytes(B, B, H, Hkv, D, table.shape[1] * page, len(prefix) * page if P else 0)
    guard = torch.full((nbytes + 4096,), 0x5A, dtype=torch.uint8, device="cuda")

    def call(ws):   # without starts, with a prefix or without: the entry below the public ones
        return api._fwd_paged(q, k, v, table, None, i32(lens), prefix, i32([P]) if P else None, None, None, None, ws)

    o, lse = call(guard[:nbytes] if nbytes else None)
    torch.cuda.synchronize()
    assert (guard[nbytes:] == 0x5A).all(), "written past the workspace"
    check(o, lse, batch(q, k, v, table, starts, lens, prefix, P), "one token")
    again = call(None)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse), "another call, other bits"


def test_one_token_nan_and_large_scores():
    """A NaN in a query or an own key is that row's alone; scores of thousands, of keys that different waves meet."""
    need_gpu()
    announce("one token NaN and large scores")
    g = torch.Generator().manual_seed(22)
    lens, P = [300, 20, 900], 3000
    q, k, v, table, starts, prefix = setup([1] * 3, lens, 8, 2, 128, 16, P, g)
    kw = dict(prefix_table=prefix, prefix_len=i32([P]))
    q *= 30
    k *= 30
    o, lse = api.attnfuse_decode_paged(q, k, v, table, i32(lens), **kw)
    check(o, lse, batch(q, k, v, table, starts, lens, prefix, P), "large")
    q[1, 2, 5] = float("nan")
    k[table[2, 40].long(), 1, 3, 7] = float("nan")
    got, gl = api.attnfuse_decode_paged(q, k, v, table, i32(lens), **kw)
    hit = torch.zeros(3, 8, dtype=torch.bool, device="cuda")
    hit[1, 2] = hit[2, 4:] = True
    assert got[hit].isnan().all() and gl[hit].isnan().all()
    assert torch.equal(got[~hit], o[~hit]) and torch.equal(gl[~hit], lse[~hit])


@pytest.mark.parametrize("n,D", [(1, 64), (1, 128), (30, 64), (30, 128), (300, 128)])
def test_keys_and_values_laid_out_otherwise(n, D):
    """K heads first, V places first, each a slice of wider pages: no stride of one is the other's."""
    need_gpu()
    announce(f"fwd_paged K and V of other strides n={n} D={D}")
    g = torch.Generator().manual_seed(23)
    Hkv, page, P, lens = 2, 32, 700, [n + 50, n]
    q, k, v, table, starts, prefix = setup([n, n], lens, 8, Hkv, D, page, P, g)
    pages = k.shape[0]
    k = torch.randn(pages, Hkv + 1, page, D + 8, generator=g).bfloat16().cuda()[:, :Hkv, :, :D]
    v = torch.randn(pages, page, Hkv + 3, D + 24, generator=g).bfloat16().cuda()[:, :, :Hkv, :D].transpose(1, 2)
    kw = dict(prefix_table=prefix, prefix_len=i32([P]))
    refs = batch(q, k, v, table, starts, lens, prefix, P)
    check(*api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), **kw), refs, "prompts")
    if n == 1:
        check(*api.attnfuse_decode_paged(q, k, v, table, i32(lens), **kw), refs, "decode")


def test_append_prompts_decode():
    """A server's run: a prefix of patches and text at positions of three axes is appended once, questions of some tokens are
    appended and attend, and then tokens one at a time."""
    need_gpu()
    announce("append, prompts, decode")
    g = torch.Generator().manual_seed(13)
    H, Hkv, D, page, P, B = 8, 2, 64, 16, 150, 3
    kc, vc = (torch.zeros(60, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    order = torch.randperm(60, generator=g).to(torch.int32)
    prefix, table = order[:10].cuda(), order[10:28].reshape(B, 6).cuda()
    cfg = dict(rope="neox", theta=10000.0, sections=(8, 12, 12), max_positions=1000, norm=False)

    def append(n, slots, pos):
        x = torch.randn(n, H + 2 * Hkv, D, generator=g).bfloat16().cuda()
        return api.attnfuse_qknorm_rope_append(x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], kc, vc, slots, positions=pos, **cfg)

    def slots_of(pages, at):
        return pages.long()[at // page] * page + at % page

    at = torch.arange(P).cuda()
    append(P, slots_of(prefix, at), torch.stack((at // 100, at % 100 // 10, at % 10)).to(torch.int32).contiguous())
    counts, lens, starts = [5, 1, 30], [5, 1, 30], [0, 5, 6, 36]
    slots = torch.cat([slots_of(table[b], torch.arange(n).cuda()) for b, n in enumerate(counts)])
    pos = torch.cat([20 + torch.arange(n) for n in counts]).to(torch.int32).cuda()
    q = append(36, slots, pos.expand(3, 36).contiguous())
    plen = i32([P])
    o, lse = api.attnfuse_fwd_paged(q, kc, vc, table, i32(starts), i32(lens), prefix_table=prefix, prefix_len=plen)
    check(o, lse, batch(q, kc, vc, table, starts, lens, prefix, P), "questions")
    for step in range(20):
        lens = [n + 1 for n in lens]
        slots = torch.stack([slots_of(table[b], torch.tensor(n - 1).cuda()) for b, n in enumerate(lens)])
        pos = torch.tensor([19 + n for n in lens], dtype=torch.int32).cuda()
        q = append(B, slots, pos.expand(3, B).contiguous())
        o, lse = api.attnfuse_decode_paged(q, kc, vc, table, i32(lens), prefix_table=prefix, prefix_len=plen)
        if step % 6 == 0:
            check(o, lse, batch(q, kc, vc, table, [0, 1, 2, 3], lens, prefix, P), f"token {step}")
    assert f64(o).isfinite().all()


@pytest.mark.parametrize("n", [1 << 17, 1 << 20])
@pytest.mark.parametrize("one", [True, False])
def test_equal_weights_of_a_long_list_in_one_share(one, n):
    """Four keys at the maximum, in the first tiles of every wave, and then n - 4 of one lower score, another in each row: the
    roundings of a running sum of equal weights all go the same way.  Scores are products of two bf16 numbers, exact in fp32."""
    need_gpu()
    announce(f"fwd_paged equal weights n={n} one={one}")
    g = torch.Generator().manual_seed(24)
    B, H, D, page = 128, 8, 128, 256
    assert api.attnfuse_fwd_paged_workspace_bytes(B, B, H, H, D, n) == 0, "more than one share"
    q, k = torch.zeros(B, H, D, dtype=torch.bfloat16), torch.zeros(2, H, page, D, dtype=torch.bfloat16)
    v = torch.randn(2, H, page, D, generator=g).bfloat16()
    q[:, :, 0] = (1 + torch.rand(B, 1, generator=g)).bfloat16()
    k[:, :, :, 0] = -(0.5 + 1.5 * torch.rand(H, generator=g)).bfloat16()[None, :, None]
    first = torch.tensor([0, 32, 64, 96])
    k[0, :, first] = 0
    table = torch.ones(B, n // page, dtype=torch.int32)
    table[:, 0] = 0
    lens = torch.full((B,), n, dtype=torch.int32).cuda()
    o, lse = api._fwd_paged(q.cuda(), k.cuda(), v.cuda(), table.cuda(), None if one else i32(list(range(B + 1))), lens, None, None,
                            1.0, None, None, None)
    low = f64(q[:, :, 0]) * f64(k[1, :, 0, 0])                       # [B, H]
    w, x = low.exp(), f64(v)
    rest = torch.ones(page, dtype=torch.bool)
    rest[first] = False

    def total(x):   # over the keys, of x [2, H, page, ...] times their weights
        at = w.reshape(B, H, *(1,) * (x.dim() - 3))
        return x[0][:, first].sum(1) + at * (x[0][:, rest].sum(1) + (n // page - 1) * x[1].sum(1))

    s = total(torch.ones(2, H, page, dtype=torch.float64))
    refs = [(slice(0, B), total(x) / s[..., None], s.log(), total(x.abs()) / s[..., None], -low)]
    check(o, lse, refs, "equal weights")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("counts,lens", [([40, 200, 130, 260], [1500, 200, 700, 700]), ([0, 700], [2000, 1000]),
                                         ([300, 1, 150, 150, 150, 90], [300, 5000, 1000, 150, 1000, -3])],
                         ids=lambda x: str(x).replace(" ", ""))
def test_joined_and_longest_first(counts, lens, D):
    """Rows enough to walk the prefix's tiles and then their own, in more workgroups than run at once: by length, which is another
    order than that of the sequences and of their numbers of rows, ties and a sequence without queries or keys among them."""
    need_gpu()
    announce(f"fwd_paged joined, longest first {counts} {lens} D={D}")
    g = torch.Generator().manual_seed(25 + len(counts))
    H, Hkv, P, page = 128, 16, 333, 16
    q, k, v, table, starts, prefix = setup(counts, lens, H, Hkv, D, page, P, g, pad=3)
    kw = dict(prefix_table=prefix, prefix_len=i32([P]))
    o, lse = api.attnfuse_fwd_paged(q, k, v, table, i32(starts), i32(lens), **kw)
    for j in (0, Hkv - 1):   # the reference of two K/V heads
        h = slice(j * H // Hkv, (j + 1) * H // Hkv)
        refs = batch(q[:, h], k[:, j:j + 1], v[:, j:j + 1], table, starts, lens, prefix, P)
        check(o[:, h], lse[:, h], refs, f"K/V head {j}")
