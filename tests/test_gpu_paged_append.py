"""Rotation and append to the paged cache, on the GPU, bit for bit against
fp32 arithmetic on the CPU (each product and sum rounded once) and the oracle's
e4m3 encoder; and a layer's whole attention half, stage by stage."""

import numpy as np
import pytest
import torch

import paper_2607_16339_amd as lc
from oracle.e4m3 import e4m3_encode
from paged_util import DEV, E4M3, Cache, attention_exact, normal

pytestmark = pytest.mark.gpu


def _tables(n, r, seed=0):
    g = torch.Generator().manual_seed(seed)
    ang = torch.rand((n, r // 2), generator=g, dtype=torch.float64) * 6.28
    return ang.cos().float(), ang.sin().float()


def _rotated(x, pos, cs, sn):
    """x [T, heads, d] fp32 on the CPU."""
    if cs is None:
        return x
    h = cs.shape[1]
    c, s = cs[pos][:, None], sn[pos][:, None]
    a, b = x[..., :h], x[..., h:2 * h]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * h:]], dim=-1)


def _bits(t):
    return t.cpu().view(torch.uint8)


class Call:
    def __init__(self, S, tokens, heads, kv, d, page, fp8, rope, max_pages=4, seed=0, rope_len=None):
        """tokens: (sequence, position) of each."""
        g = torch.Generator().manual_seed(seed)
        self.T, self.fp8, self.page, self.kv, self.heads, self.d, self.S = len(tokens), fp8, page, kv, heads, d, S
        self.num_pages, self.max_pages = S * max_pages + 2, max_pages
        self.qkv = normal(g, (self.T, (heads + 2 * kv) * d), 2.0)
        self.seq = torch.tensor([t[0] for t in tokens], dtype=torch.int32)
        self.pos = torch.tensor([t[1] for t in tokens], dtype=torch.int32)
        self.table = torch.randperm(self.num_pages, generator=g)[: S * max_pages].view(S, max_pages).to(torch.int32)
        self.rope_len = page * max_pages if rope_len is None else rope_len
        self.cs, self.sn = _tables(self.rope_len, rope, seed) if rope else (None, None)
        shape = (self.num_pages, kv, page, d)
        if fp8:
            self.k, self.v = (torch.randint(0, 127, shape, generator=g, dtype=torch.uint8) for _ in range(2))
            self.ks, self.vs = (torch.rand(shape[:3], generator=g) for _ in range(2))
        else:
            self.k, self.v = normal(g, shape), normal(g, shape)
            self.ks = self.vs = None
        self.q = torch.full((self.T, heads, d), 9.0, dtype=torch.bfloat16)

    def want(self):
        q, k, v = self.q.clone(), self.k.clone(), self.v.clone()
        ks, vs = (None, None) if self.ks is None else (self.ks.clone(), self.vs.clone())
        x = self.qkv.float().view(self.T, -1, self.d)
        turned = self.heads + self.kv
        safe = self.pos.long().clamp(0, self.rope_len - 1)
        y = torch.cat([_rotated(x[:, :turned], safe, self.cs, self.sn), x[:, turned:]], dim=1)
        for t in range(self.T):
            s, p = int(self.seq[t]), int(self.pos[t])
            if not 0 <= s < self.S or not 0 <= p < self.page * self.max_pages:
                continue
            if self.cs is not None and p >= self.rope_len:
                continue
            at, slot = int(self.table[s, p // self.page]), p % self.page
            if not 0 <= at < self.num_pages:
                continue
            q[t] = y[t, : self.heads].to(torch.bfloat16)
            for cache, scale, val in ((k, ks, y[t, self.heads:turned]), (v, vs, y[t, turned:])):
                if self.fp8:
                    sc = val.abs().amax(dim=-1) / 448.0
                    quo = val / torch.where(sc == 0, torch.ones_like(sc), sc)[:, None]
                    cache[at, :, slot] = torch.from_numpy(e4m3_encode(quo.numpy().astype(np.float32)).astype(np.uint8))
                    cache[at, :, slot][sc == 0] = 0
                    scale[at, :, slot] = sc
                else:
                    cache[at, :, slot] = val.to(torch.bfloat16)
        return [q, k, v] + ([] if ks is None else [ks, vs])

    def run(self, stream=None):
        dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        out = [dev(t) for t in (self.q, self.k, self.v, self.ks, self.vs)]
        lc.lacache_paged_append(dev(self.qkv), dev(self.seq), dev(self.pos), dev(self.cs), dev(self.sn),
                                dev(self.table), *out[:3], *out[3:], stream=stream)
        torch.cuda.synchronize()
        return [t for t in out if t is not None]

    def check(self, what):
        for name, got, want in zip(("q", "k", "v", "k_scale", "v_scale"), self.run(), self.want()):
            assert torch.equal(_bits(got), _bits(want)), (what, name)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,rope", [(128, 128), (64, 64), (128, 64), (128, 16), (64, 48), (128, 0)])
@pytest.mark.parametrize("heads,kv,page", [(4, 4, 16), (32, 8, 64), (3, 1, 256), (7, 7, 32)])
def test_append_exact(heads, kv, page, d, rope, fp8):
    toks = [(0, 0), (1, 5), (2, page), (0, 1), (1, 4 * page - 1), (2, 3 * page + 7)]
    Call(3, toks, heads, kv, d, page, fp8, rope, seed=heads + rope).check("heads %d/%d rope %d" % (heads, kv, rope))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [1, 2, 63, 1000, 3000])
def test_numbers_of_tokens(T, fp8):
    per = -(-T // 5)
    toks = [(i // per, i % per) for i in range(T)]
    Call(5, toks, 8, 2, 128, 64, fp8, 128, max_pages=max(1, -(-per // 64)), seed=T).check("T %d" % T)


@pytest.mark.parametrize("fp8", [False, True])
def test_skipped_tokens_leave_everything_as_it_was(fp8):
    toks = [(-1, 3), (0, -1), (2, 3), (0, 64), (1, 40), (1, 63), (0, 2), (2 ** 31 - 1, 0), (0, 2 ** 31 - 1), (0, 17)]
    c = Call(2, toks, 4, 2, 128, 16, fp8, 128, seed=3, rope_len=50)  # position 63 has no row of the tables
    c.table[0, 1] = -1  # position 17
    c.table[1, 2] = c.num_pages  # position 40
    c.check("skipped")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,kv,d", [(32, 8, 128), (16, 8, 64), (1, 1, 64), (9, 3, 128)])
def test_skipped_tokens_among_others(heads, kv, d, fp8):
    # whole workgroups of a token, and workgroups of several tokens
    toks = [(-1 if i % 3 == 1 else i % 2, -1 if i % 7 == 2 else i // 2) for i in range(101)]
    c = Call(2, toks, heads, kv, d, 16, fp8, d, seed=heads, rope_len=45)
    c.table[1, 1] = -1
    c.check("skipped among others")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,heads,kv,d", [(1501, 1, 1, 64), (701, 4, 1, 64), (777, 5, 5, 128), (1100, 14, 2, 64), (600, 24, 12, 128)])
def test_many_tokens_of_few_heads(T, heads, kv, d, fp8):
    Call(3, [(i % 3, i // 3) for i in range(T)], heads, kv, d, 128, fp8, 32, max_pages=4, seed=T).check("T %d heads %d" % (T, heads))


def test_zeros_and_values_that_are_no_numbers():
    c = Call(1, [(0, i) for i in range(6)], 2, 1, 64, 16, True, 0, seed=4)
    x = c.qkv.view(6, 4, 64)
    x[0] = 0.0
    x[1, :, 3] = 1e-38
    x[2] = 3.3e38
    c.check("zeros, tiny and huge values")
    x[3, 2, 7], x[4, 3, 0], x[5, 0, 1] = float("nan"), float("inf"), float("-inf")
    got = c.run()
    q, k, v, ks, vs = (t.cpu() for t in got)
    at = int(c.table[0, 0])
    # the number that is none makes its own vector's values none, the others stay
    kd = k[at, 0].view(E4M3).float() * ks[at, 0][:, None]
    vd = v[at, 0].view(E4M3).float() * vs[at, 0][:, None]
    assert not bool(torch.isfinite(kd[3]).all()) and bool(torch.isfinite(kd[[0, 1, 2, 4, 5]]).all())
    assert not bool(torch.isfinite(vd[4]).all()) and bool(torch.isfinite(vd[[0, 1, 2, 3, 5]]).all())
    assert float(q[5, 0, 1]) == float("-inf")


def test_offsets_beyond_32_bits():
    page, kv, d = 256, 8, 128
    num = (5 << 30) // (page * kv * d * 2) + 2
    k = torch.zeros((num, kv, page, d), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    c = Call(1, [(0, 3), (0, 300)], 8, kv, d, page, False, 128, seed=5)
    table = torch.tensor([[num - 1, num - 2, -1, -1]], dtype=torch.int32, device=DEV)
    q = torch.empty((2, 8, d), dtype=torch.bfloat16, device=DEV)
    lc.lacache_paged_append(c.qkv.to(DEV), c.seq.to(DEV), c.pos.to(DEV), c.cs.to(DEV), c.sn.to(DEV), table, q, k, v)
    torch.cuda.synchronize()
    want = c.want()
    for got, w in ((k, want[1]), (v, want[2])):
        assert torch.equal(_bits(got[num - 1, :, 3]), _bits(w[int(c.table[0, 0]), :, 3]))
        assert torch.equal(_bits(got[num - 2, :, 44]), _bits(w[int(c.table[0, 1]), :, 44]))
        assert int(torch.count_nonzero(got[: num - 2])) == 0


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("nq", [1, 32])
def test_attention_half_of_a_layer(nq, fp8):
    """QKV product with bias -> append -> attention -> output product added to the residual stream
    in place -> the FFN with its AddNorm: eagerly, and as a graph replayed over a changed input."""
    H, heads, kv, d, page, I = 512, 8, 2, 64, 16, 512
    lens = [nq, 40 + nq, 300]
    S = len(lens)
    cache = Cache(lens, heads, kv, d, page, fp8, seed=6, max_pages=20)
    g = torch.Generator().manual_seed(7)
    T = S * nq
    x0, w_qkv, b_qkv = normal(g, (T, H)), normal(g, ((heads + 2 * kv) * d, H), 0.05), normal(g, ((heads + 2 * kv) * d,))
    w_o, nw = normal(g, (H, heads * d), 0.05), normal(g, (H,), 0.1)
    wgu, wd = normal(g, (2 * I, H), 0.05), normal(g, (H, I), 0.05)
    x0, w_qkv, b_qkv, w_o, nw, wgu, wd = (t.to(DEV) for t in (x0, w_qkv, b_qkv, w_o, nw, wgu, wd))
    gu, dn = lc.quantize_weights(wgu), lc.quantize_weights(wd)
    cs, sn = (t.to(DEV) for t in _tables(page * 20, d, 8))
    seq = torch.arange(S, dtype=torch.int32, device=DEV).repeat_interleave(nq)
    pos = (cache.lens[:, None] - nq + torch.arange(nq, dtype=torch.int32, device=DEV)).reshape(-1).contiguous()
    x = x0.clone()
    qkv = torch.empty((T, (heads + 2 * kv) * d), dtype=torch.bfloat16, device=DEV)
    q = torch.empty((S, nq, heads, d), dtype=torch.bfloat16, device=DEV)
    o, out, zero = torch.empty_like(q), torch.empty_like(x), torch.zeros_like(x)

    def step():
        lc.lacache_linear_act_bf16(x, w_qkv, qkv, bias=b_qkv)
        lc.lacache_paged_append(qkv, seq, pos, cs, sn, cache.table, q.view(T, heads, d), cache.k, cache.v,
                                cache.k_scale, cache.v_scale)
        lc.lacache_paged_attention(q, cache.k, cache.v, cache.table, cache.lens, o, k_scale=cache.k_scale,
                                   v_scale=cache.v_scale, causal=nq == 1)
        lc.lacache_linear_act_bf16(o.view(T, heads * d), w_o, x, residual=x)
        lc.lacache_ffn_fp8_addnorm(x, zero, nw, *gu, *dn, out)

    step()
    torch.cuda.synchronize()
    # each stage against its own inputs
    want = x0.double() @ w_qkv.double().t().contiguous() + b_qkv.double()
    assert bool(((qkv.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())
    ref = attention_exact(cache, q, nq == 1)
    assert bool(((o.double() - ref[0]).abs() <= ref[2]).all())
    want = o.view(T, -1).double() @ w_o.double().t().contiguous() + x0.double()
    assert bool(((x.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())
    ffn = lc.ffn_fp8(x, nw, *gu, *dn)
    assert torch.equal(_bits(ffn), _bits(out))
    eager = [t.clone() for t in (qkv, q, o, x, out)]
    graph = torch.cuda.CUDAGraph()
    x.copy_(x0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for other in (False, True, False):
        x.copy_(x0 * 0.5 if other else x0)
        graph.replay()
        torch.cuda.synchronize()
        same = [torch.equal(_bits(a), _bits(b)) for a, b in zip((qkv, q, o, x, out), eager)]
        assert all(same) if not other else not any(same)
