"""Attention over the paged cache at the places where a key can be lost or a
value leak: rows that every score hides, values that are no numbers in causal
tiles. Each form of the kernel is reached by its number of rows per KV head and
by its number of sequences (FORMS)."""

import math

import pytest
import torch

import paper_2607_16339_amd as lc
from paged_util import DEV, Cache, attend, normal

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
# (nq, heads, kv): 8, 16 rows per KV head (one row tile), 40 (two), 80 and 208 (wavefronts that split the rows)
FORMS = [(8, 1, 1), (8, 4, 2), (20, 2, 1), (40, 2, 1), (26, 16, 2)]


def _q(c, nq, seed=1, std=1.5):
    return normal(torch.Generator().manual_seed(seed), (c.S, nq, c.heads, c.d), std).to(DEV)


def _bits(t):
    return t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32)


def _place(c, s, key):
    return int(c.table[s, key // c.page]), key % c.page


def _put_value(c, s, key, head, dim, x):
    """Value `key` of sequence s in dimension `dim` becomes x (of an e4m3 cache: NaN)."""
    page, slot = _place(c, s, key)
    if c.fp8:
        c.v.view(torch.uint8)[page, head, slot, dim] = 0x7F
    else:
        c.v[page, head, slot, dim] = x


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,heads,kv", FORMS)
def test_rows_whose_scores_are_all_minus_infinity_take_no_value(nq, heads, kv, d, fp8):
    """o = 0 and lse = -inf whatever the values hold, of whole sequences and of cut ones."""
    lens = [60, 4500, 333]
    c = Cache(lens, heads, kv, d, 16, fp8, seed=nq + d)
    q = _q(c, nq).abs().clamp_min(0.125)  # (-inf times 0 would be none)
    for s in (0, 1):
        pages = c.table[s, : -(-lens[s] // 16)].long()
        if fp8:
            c.k.view(torch.uint8)[pages] = 0x38  # 1.0
            c.k_scale[pages] = -INF
        else:
            c.k[pages] = -INF
        for key, x in ((3, INF), (lens[s] // 2, NAN), (lens[s] - 1, -INF)):
            for h in range(kv):
                _put_value(c, s, key, h, 7, x)
    o, lse = attend(c, q, False)
    torch.cuda.synchronize()
    assert bool((o[:2] == 0).all()) and bool((lse[:2] == -math.inf).all())
    assert bool(torch.isfinite(o[2].float()).all()) and bool(torch.isfinite(lse[2]).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,heads,kv", FORMS)
@pytest.mark.parametrize("length,key", [(128, 125), (128, 67), (4992, 4989)])
def test_values_of_hidden_keys_move_no_bit(length, key, nq, heads, kv, d, fp8):
    """A value that is no number late in a tile: causal rows before it keep every bit, although
    they see other keys of its tile; rows that see it keep every other dimension's."""
    c = Cache([length, 70], heads, kv, d, 16, fp8, seed=length + d)
    q = _q(c, nq)
    want, wl = attend(c, q, True)
    for dim, x in ((5, NAN), (d - 2, INF), (5, -INF)):
        old = c.v.view(torch.uint8).clone()
        for h in range(kv):
            _put_value(c, 0, key, h, dim, x)
        o, lse = attend(c, q, True)
        torch.cuda.synchronize()
        c.v.view(torch.uint8).copy_(old)
        sees = [t for t in range(nq) if key <= length - nq + t]
        assert torch.equal(_bits(lse), _bits(wl)), (dim, x)
        keep = torch.ones(o.shape, dtype=torch.bool, device=DEV)
        keep[0, sees, :, dim] = False
        assert torch.equal(_bits(o)[keep], _bits(want)[keep]), (dim, x)
        assert not bool(torch.isfinite(o.float())[~keep].any()), (dim, x)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,heads,kv", FORMS)
def test_first_call_is_captured_where_no_sequence_can_be_cut(nq, heads, kv, d, fp8):
    """A table of two tiles: the call needs no workspace, so the library need not have one."""
    c = Cache([60, 1, 64], heads, kv, d, 16, fp8, seed=nq + d)
    q = _q(c, nq)
    o, lse = torch.empty_like(q), torch.empty(q.shape[:3], dtype=torch.float32, device=DEV)
    torch.cuda.synchronize()
    lc.lacache_release_workspace()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lc.lacache_paged_attention(q, c.k, c.v, c.table, c.lens, o, lse=lse, k_scale=c.k_scale, v_scale=c.v_scale,
                                   causal=True)
    want, wl = attend(c, q, True)
    for _ in range(3):
        o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(_bits(o), _bits(want)) and torch.equal(_bits(lse), _bits(wl))


def test_library_workspace_is_bounded_by_the_table():
    """32 tokens of 32 heads over 8 KV heads and a table of 1024 keys: at most 16 pieces of 8 KV
    heads with 128 rows, 8.5 MB, where tables without end would need 136."""
    c = Cache([1000], 32, 8, 128, 16, False, seed=24, max_pages=64)
    q = _q(c, 32)
    o = torch.empty_like(q)
    torch.cuda.synchronize()
    lc.lacache_release_workspace()
    free = torch.cuda.mem_get_info()[0]
    lc.lacache_paged_attention(q, c.k, c.v, c.table, c.lens, o)
    torch.cuda.synchronize()
    taken = free - torch.cuda.mem_get_info()[0]
    n = lc.lacache_paged_attention_workspace_bytes(1, 32, 32, 8, 128)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    want, _ = attend(c, q, False, workspace=ws)
    torch.cuda.synchronize()
    assert n > 100 << 20 and 0 < taken <= 16 << 20, (n, taken)
    assert torch.equal(_bits(o), _bits(want))
