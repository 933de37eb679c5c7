"""Attention of new tokens over the paged cache, on the GPU, against its
definition in 64 bits (paged_util: the tolerance is derived there). Every place
of the cache that no token of a sequence fills holds NaN or infinity, so a read
that reaches the result shows."""

import math

import pytest
import torch

import paper_2607_16339_amd as lc
from paged_util import DEV, E4M3, Cache, attend, attention_exact, check_attention, normal

pytestmark = pytest.mark.gpu


def _q(c, nq, seed=1, std=1.5):
    return normal(torch.Generator().manual_seed(seed), (c.S, nq, c.heads, c.d), std).to(DEV)


def _bits(t):
    return t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32)


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_lengths_around_every_border(page, d, fp8):
    c = Cache(EDGES, 8, 2, d, page, fp8, seed=page + d)
    check_attention(c, _q(c, 1), True, what="page %d d %d fp8 %d" % (page, d, fp8))


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (3, 1), (8, 1), (7, 1), (32, 8), (16, 1), (17, 1), (40, 1), (36, 2)])
@pytest.mark.parametrize("fp8", [False, True])
def test_head_layouts(heads, kv, fp8):
    c = Cache([1, 100, 333], heads, kv, 128, 16, fp8, seed=heads)
    check_attention(c, _q(c, 1), False, what="heads %d kv %d" % (heads, kv))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("nq,heads,kv", [(2, 4, 1), (5, 6, 2), (8, 2, 2), (16, 4, 1), (32, 8, 8), (33, 2, 2), (64, 8, 2),
                                         (32, 32, 4)])
@pytest.mark.parametrize("fp8", [False, True])
def test_blocks_of_tokens(nq, heads, kv, causal, fp8):
    # lengths below nq: causal tokens before the first key see nothing
    c = Cache([0, 1, nq - 1, nq, nq + 1, 70, 300], heads, kv, 128, 16, fp8, seed=nq)
    check_attention(c, _q(c, nq), causal, what="nq %d heads %d/%d causal %d" % (nq, heads, kv, causal))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,heads,kv", [([40001], 8, 2), ([20000, 5, 3000, 0, 777], 4, 1), ([2000] * 9, 32, 32),
                                           (list(range(1, 700, 9)), 8, 4)])
def test_long_and_ragged(lens, heads, kv, d, fp8):
    c = Cache(lens, heads, kv, d, 16, fp8, seed=len(lens))
    check_attention(c, _q(c, 1), True, what="lens %s.. d %d fp8 %d" % (lens[:3], d, fp8))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,heads,kv,page,causal,lens", [
    (9, 8, 2, 16, True, [3000, 40, 0, 700]),      # 36 rows per KV head
    (16, 4, 1, 64, False, [1500, 16, 33]),        # 64
    (13, 16, 2, 32, True, [2500, 13, 6]),         # 104
    (32, 8, 2, 256, False, [1000, 513]),          # 128
    (26, 16, 2, 16, True, [1900, 1027, 30]),      # 208: two row tiles, the second not full
    (64, 6, 1, 128, False, [700]),                # 384
])
def test_many_rows_over_long_sequences(nq, heads, kv, page, causal, lens, d, fp8):
    c = Cache(lens, heads, kv, d, page, fp8, seed=nq * heads)
    check_attention(c, _q(c, nq), causal, what="nq %d heads %d/%d d %d" % (nq, heads, kv, d))


def test_many_rows_in_one_long_sequence():
    # several pages of page numbers, and pieces of several
    c = Cache([20011], 8, 1, 128, 16, False, seed=77)
    check_attention(c, _q(c, 12), True, what="96 rows over 20011 keys")


def test_many_sequences():
    # more sequences than a wavefront has lanes
    lens = [(37 * i) % 200 for i in range(700)]
    c = Cache(lens, 2, 1, 64, 16, False, seed=5)
    check_attention(c, _q(c, 1), True, what="700 sequences")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,heads", [(1, 16), (1, 64), (20, 16), (40, 16)])
def test_more_sequences_than_the_chip_takes_at_once(nq, heads, d, fp8):
    # of every length around a border, and one of several pieces
    c = Cache(EDGES + [5000] + EDGES, heads, 16, d, 32, fp8, seed=heads + nq)
    check_attention(c, _q(c, nq), True, what="nq %d heads %d d %d fp8 %d" % (nq, heads, d, fp8))


@pytest.mark.parametrize("scale", [0.0, 1e-3, 1.0])
def test_scales_of_the_scores(scale):
    c = Cache([1, 90, 200], 4, 2, 128, 32, False, seed=3)
    check_attention(c, _q(c, 3, std=0.5), False, scale=scale, what="scale %g" % scale)


@pytest.mark.parametrize("fp8", [False, True])
def test_large_scores(fp8):
    """Scores of several hundred: a running maximum that climbs through the keys."""
    c = Cache([257, 1000], 4, 1, 128, 16, fp8, seed=9, kstd=20.0)
    check_attention(c, _q(c, 2, std=4.0), True, what="large scores")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal", [False, True])
def test_bad_pages_and_lengths(causal, fp8):
    """Keys on pages of no number are left out; lengths are held to the table's capacity."""
    c = Cache([300, 200, 100, 64], 4, 2, 128, 16, fp8, seed=11)
    c.table[0, 3], c.table[0, 7], c.table[1, 0] = -1, c.num_pages, 2 ** 31 - 1
    c.table[2] = -1  # no key at all
    c.lens[3] = -5
    o, lse = check_attention(c, _q(c, 5), causal, what="bad pages")
    assert bool((o[2] == 0).all()) and bool((lse[2] == -math.inf).all()) and bool((o[3] == 0).all())
    full = Cache([96, 96], 4, 2, 128, 16, fp8, seed=12)
    want = attend(full, _q(full, 5), causal)
    full.lens[0], full.lens[1] = 2 ** 31 - 1, 97  # the table holds 6 pages
    got = attend(full, _q(full, 5), causal)
    assert torch.equal(_bits(got[0]), _bits(want[0])) and torch.equal(_bits(got[1]), _bits(want[1]))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("nq,heads", [(6, 4), (40, 1), (40, 2)])
def test_hidden_keys_do_not_reach_a_row(bad, nq, heads, fp8):
    """A key or value that is no number changes only the rows that see it, causal rows before it not."""
    c = Cache([100], heads, 1, 128, 16, fp8, seed=13)
    q = _q(c, nq)
    want, wl = attend(c, q, True)
    at = 100 - 3  # seen by the last three tokens
    page, slot = int(c.table[0, at // 16]), at % 16
    for which in ("k", "v"):
        x = getattr(c, which)
        old = x.view(torch.uint8).clone()
        if fp8:
            x.view(torch.uint8)[page, 0, slot, 5] = 0x7F
            sc = getattr(c, which + "_scale")
            olds = sc.clone()
            if bad == bad:
                x.view(torch.uint8)[page, 0, slot, 5] = 0x38
                sc[page, 0, slot] = bad
        else:
            x[page, 0, slot, 5] = bad
        o, lse = attend(c, q, True)
        torch.cuda.synchronize()
        assert torch.equal(_bits(o[:, :-3]), _bits(want[:, :-3])), which
        assert torch.equal(_bits(lse[:, :-3]), _bits(wl[:, :-3])), which
        if which == "v":
            assert not bool(torch.isfinite(o[:, -3:].float()).all())
            if not fp8:  # the other dimensions are as they were
                keep = [i for i in range(128) if i != 5]
                assert bool(torch.isfinite(o[..., keep].float()).all())
        x.view(torch.uint8).copy_(old)
        if fp8:
            sc.copy_(olds)


def test_rows_whose_scores_are_all_minus_infinity():
    c = Cache([5, 60], 2, 1, 64, 16, False, seed=14)
    q = _q(c, 1).abs()
    c.k[c.table[0, 0].long(), :, :5] = float("-inf")
    o, lse = attend(c, q, False)
    torch.cuda.synchronize()
    assert bool((o[0] == 0).all()) and bool((lse[0] == -math.inf).all()) and bool(torch.isfinite(o[1].float()).all())


@pytest.mark.parametrize("fp8", [False, True])
def test_offsets_beyond_32_bits(fp8):
    """Pages more than 4 GiB into the cache."""
    page, kv, d = 256, 8, 128
    num = (5 << 30) // (page * kv * d) + 2
    dt = torch.uint8 if fp8 else torch.bfloat16
    c = Cache([300, 77], 16, kv, d, page, fp8, seed=15)
    big = Cache([300, 77], 16, kv, d, page, fp8, seed=15)
    for name in ("k", "v"):
        x = torch.zeros((num, kv, page, d), dtype=dt, device=DEV)
        x[-c.num_pages:] = getattr(c, name).view(dt)
        setattr(big, name, x.view(E4M3) if fp8 else x)
        if fp8:
            s = torch.zeros((num, kv, page), dtype=torch.float32, device=DEV)
            s[-c.num_pages:] = getattr(c, name + "_scale")
            setattr(big, name + "_scale", s)
    big.table = torch.where(c.table < 0, c.table, c.table + (num - c.num_pages))
    big.num_pages = num
    q = _q(c, 2)
    want, got = attend(c, q, True), attend(big, q, True)
    torch.cuda.synchronize()
    assert torch.equal(_bits(want[0]), _bits(got[0])) and torch.equal(_bits(want[1]), _bits(got[1]))


def test_shared_pages_and_shared_inputs():
    """Sequences that share a prefix's pages; the same sequence twice gives the same bytes."""
    c = Cache([200, 200], 8, 2, 128, 16, False, seed=16)
    c.table[1] = c.table[0]
    q = _q(c, 3)
    q[1] = q[0]
    o, lse = attend(c, q, True)
    torch.cuda.synchronize()
    assert torch.equal(_bits(o[0]), _bits(o[1])) and torch.equal(_bits(lse[0]), _bits(lse[1]))


def test_same_bytes_again_without_lse_and_with_a_workspace():
    c = Cache([5000, 1, 40, 900], 16, 4, 128, 32, True, seed=17)
    q = _q(c, 4)
    o, lse = attend(c, q, True)
    o2, none = attend(c, q, True, lse=False)
    n = lc.lacache_paged_attention_workspace_bytes(c.S, 4, 16, 4, 128)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    o3, l3 = attend(c, q, True, workspace=ws)
    torch.cuda.synchronize()
    assert none is None and torch.equal(_bits(o), _bits(o2)) and torch.equal(_bits(o), _bits(o3))
    assert torch.equal(_bits(lse), _bits(l3))
    with pytest.raises(lc.LacacheError) as e:
        attend(c, q, True, workspace=ws[: n - 256] if n > 256 else ws[:0])
    assert e.value.status == lc.LACACHE_ERR_INVALID_ARG


def test_nothing_is_written_around_the_outputs():
    c = Cache([77, 0, 300], 6, 2, 64, 16, False, seed=18)
    q = _q(c, 3)
    n = q.numel()
    buf = torch.full((n + 512,), 3.0, dtype=torch.bfloat16, device=DEV)
    o = buf[256:256 + n].view(q.shape)
    lbuf = torch.full((c.S * 18 + 128,), 3.0, dtype=torch.float32, device=DEV)
    lse = lbuf[64:64 + c.S * 18].view(c.S, 3, 6)
    lc.lacache_paged_attention(q, c.k, c.v, c.table, c.lens, o, lse=lse, causal=True)
    torch.cuda.synchronize()
    assert bool((buf[:256] == 3).all()) and bool((buf[256 + n:] == 3).all())
    assert bool((lbuf[:64] == 3).all()) and bool((lbuf[64 + c.S * 18:] == 3).all())
    ref = attention_exact(c, q, True)
    assert bool(((o.double() - ref[0]).abs() <= ref[2]).all())


def test_captured_and_replayed_with_growing_lengths():
    """A graph of one decoding step, replayed while the lengths grow on the device."""
    c = Cache([1000, 37, 400], 8, 2, 128, 16, False, seed=19)
    q = _q(c, 1)
    full = c.lens.clone()
    ws = torch.empty(lc.lacache_paged_attention_workspace_bytes(3, 1, 8, 2, 128), dtype=torch.uint8, device=DEV)
    attend(c, q, True, workspace=ws)
    torch.cuda.synchronize()
    o = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lc.lacache_paged_attention(q, c.k, c.v, c.table, c.lens, o, causal=True, workspace=ws)
    for sub in (30, 0, 7, 30, 1):
        c.lens.copy_(full - sub)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        want, _ = attend(c, q, True)
        torch.cuda.synchronize()
        assert torch.equal(_bits(got), _bits(want)), sub


@pytest.mark.parametrize("nq", [1, 12, 20])  # 4, 48 and 80 rows per KV head
def test_captured_and_replayed_with_cuts_that_move(nq):
    """Two graphs on one workspace; their sequences go from many pieces to one and back."""
    c = Cache([9000, 2500, 64], 8, 2, 128, 16, False, seed=23)
    q, full = _q(c, nq), c.lens.clone()
    ws = torch.empty(lc.lacache_paged_attention_workspace_bytes(3, nq, 8, 2, 128), dtype=torch.uint8, device=DEV)
    attend(c, q, True, workspace=ws)
    torch.cuda.synchronize()
    outs, graphs = [torch.empty_like(q) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    for o, graph, causal in zip(outs, graphs, (True, False)):
        with torch.cuda.graph(graph):
            lc.lacache_paged_attention(q, c.k, c.v, c.table, c.lens, o, causal=causal, workspace=ws)
    for lens in (full.tolist(), [100, 2500, 0], [9000, 0, 64], [1, 1, 1], [4000, 2000, 33], full.tolist()):
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for o, causal in zip(outs, (True, False)):
            got = o.clone()
            want, _ = attend(c, q, causal)
            torch.cuda.synchronize()
            assert torch.equal(_bits(got), _bits(want)), (lens, causal)


@pytest.mark.parametrize("nq,heads,kv", [(1, 8, 2), (20, 8, 2), (40, 2, 2), (20, 32, 8)])
@pytest.mark.parametrize("S,longest", [(1, 20000), (3, 1100), (20, 1100), (50, 140), (120, 140), (127, 2100)])
def test_workspace_is_as_large_as_it_is_said_to_be(S, longest, nq, heads, kv):
    """What lies behind the workspace stays; lengths just above those that are not cut."""
    c = Cache([longest - (i % 5) * (longest // 50) for i in range(S)], heads, kv, 64, 16, True, seed=S)
    q = _q(c, nq)
    n = lc.lacache_paged_attention_workspace_bytes(S, nq, heads, kv, 64)
    buf = torch.full((n + (1 << 20),), 0xAB, dtype=torch.uint8, device=DEV)
    o, _ = attend(c, q, False, workspace=buf[:n])
    want, _ = attend(c, q, False)
    torch.cuda.synchronize()
    assert bool((buf[n:] == 0xAB).all()) and torch.equal(_bits(o), _bits(want))


def test_two_streams_with_their_own_workspaces():
    cs = [Cache([3000, 100 + i], 8, 2, 128, 16, False, seed=20 + i) for i in range(2)]
    qs = [_q(c, 1, seed=i) for i, c in enumerate(cs)]
    want = [attend(c, q, True)[0].clone() for c, q in zip(cs, qs)]
    n = lc.lacache_paged_attention_workspace_bytes(2, 1, 8, 2, 128)
    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in cs]
    outs = [torch.empty_like(q) for q in qs]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in cs]
    for _ in range(20):
        for c, q, w, o, s in zip(cs, qs, ws, outs, st):
            lc.lacache_paged_attention(q, c.k, c.v, c.table, c.lens, o, causal=True, workspace=w, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(_bits(o), _bits(w))


def test_no_sequences():
    c = Cache([10], 4, 2, 64, 16, False)
    z = torch.empty((0, 1, 4, 64), dtype=torch.bfloat16, device=DEV)
    lc.lacache_paged_attention(z, c.k, c.v, c.table[:0].contiguous(), c.lens[:0].contiguous(), torch.empty_like(z))
    torch.cuda.synchronize()
