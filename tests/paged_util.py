"""Inputs of the paged cache's tests and the same operators in 64 bits, written
from their definitions in elementary torch operations.

Tolerance of the attention (derived, element by element). u = 2^-24. A score is
a sum of d exact products in fp32 (any order: d u sum|q k|) times one or two
factors (3 u |s|); with the exponential's argument in fp32 and the hardware
exp2 (2 u relative) a p is off by e_p = (d + 4) u scale sum|q k| + 4 u |s - m| + 4 u,
relatively. P enters the value product as two bf16 terms (2^-16 relative) and
the n products are summed in fp32 (n u of sum p |v|), as is l. Splitting the
keys multiplies a part by another exponential (4 u + 2 u |s - m|). The base may lie
up to 8 (in powers of 2) below m: an argument's rounding then grows by 8 u, a p by
8 u ln 2, the quotient of two sums by less than 2^-20, the last term. So
  |o - ref| <= 2^-8 |ref| + (2 max e_p + 2^-16 + 2 n u + 2^-20) sum p |v| / l,
the first term the one rounding to bf16, and
  |lse - ref| <= max e_p + n u + 2^-20 + 2^-22 |ref|.
"""

import math

import torch

import paper_2607_16339_amd as lc

DEV = "cuda:0"
U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn


def normal(g, shape, std=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float32) * std).to(torch.bfloat16)


def quantize(x):
    """e4m3 codes (as float8) and scales max|x| / 448 of fp32 vectors."""
    s = x.abs().amax(dim=-1) / 448.0
    return (x / torch.where(s == 0, torch.ones_like(s), s)[..., None]).to(E4M3), s


class Cache:
    """Pages on the GPU, with NaN everywhere that no token of a sequence is placed."""

    def __init__(self, lens, heads, kv, d, page, fp8, seed=0, max_pages=None, extra=3, kstd=1.5, device=DEV):
        g = torch.Generator().manual_seed(seed)
        S = len(lens)
        need = [max(0, -(-n // page)) for n in lens]
        self.max_pages = max(1, max(need, default=1)) if max_pages is None else max_pages
        self.num_pages = max(1, sum(need) + extra)
        self.heads, self.kv, self.d, self.page, self.fp8, self.S = heads, kv, d, page, fp8, S
        order = torch.randperm(self.num_pages, generator=g).tolist()
        # entries that no sequence reaches hold numbers of no page
        self.table = torch.full((S, self.max_pages), -7, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            for p in range(min(n, self.max_pages)):
                self.table[s, p] = order[at]
                at += 1
        shape = (self.num_pages, kv, page, d)
        k, v = normal(g, shape, kstd), normal(g, shape)
        used = torch.zeros((self.num_pages, page), dtype=torch.bool)
        for s, n in enumerate(lens):
            for p in range(min(need[s], self.max_pages)):
                used[self.table[s, p], : min(page, n - p * page)] = True
        hole = ~used[:, None, :, None].expand(shape)
        self.k_scale = self.v_scale = None
        if fp8:
            (k, ks), (v, vs) = quantize(k.float()), quantize(v.float())
            hs = ~used[:, None, :].expand(shape[:3])
            ks[hs] = float("nan")
            vs[hs] = float("inf")
            kb, vb = k.view(torch.uint8).clone(), v.view(torch.uint8).clone()
            kb[hole] = 0x7F
            vb[hole] = 0xFF
            k, v = kb.view(E4M3), vb.view(E4M3)
            self.k_scale, self.v_scale = ks.to(device), vs.to(device)
        else:
            k[hole] = float("nan")
            v[hole] = float("-inf")
        self.k, self.v = k.to(device), v.to(device)
        self.table = self.table.to(device)
        self.lens = torch.tensor(lens, dtype=torch.int32).to(device)

    def values(self, s, n):
        """Keys and values [kv, n, d] of sequence s in 64 bits."""
        out = []
        at = self.table[s].long()[: -(-n // self.page)]
        ok = (at >= 0) & (at < self.num_pages)
        at = torch.where(ok, at, torch.zeros_like(at))
        for x, sc in ((self.k, self.k_scale), (self.v, self.v_scale)):
            x = x.view(torch.uint8)[at].view(x.dtype).double()
            if sc is not None:
                x = x * sc[at].double()[..., None]
            out.append(x.transpose(0, 1).reshape(self.kv, -1, self.d)[:, :n])
        return out + [ok.repeat_interleave(self.page)[:n]]


def attention_exact(c, q, causal, scale=None):
    """(o, lse, tolerance of o, tolerance of lse) in 64 bits."""
    S, nq, heads, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    G = heads // c.kv
    o = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device=q.device)
    to, tl = torch.zeros_like(o), torch.zeros_like(lse)
    for s in range(S):
        n = min(max(int(c.lens[s]), 0), c.max_pages * c.page)
        if n == 0:
            continue
        k, v, ok = c.values(s, n)
        for t in range(nq):
            see = ok.clone()
            if causal:
                see[max(0, n - nq + t + 1):] = False
            if not bool(see.any()):
                continue
            qd = q[s, t].double().view(c.kv, G, d)
            kk, vv = k[:, see].contiguous(), v[:, see].contiguous()
            x = scale * torch.bmm(qd, kk.transpose(1, 2).contiguous())
            mag = scale * torch.bmm(qd.abs(), kk.abs().transpose(1, 2).contiguous())
            m = x.amax(dim=2, keepdim=True)
            p = torch.exp(x - m)
            l = p.sum(dim=2, keepdim=True)
            o[s, t] = (torch.bmm(p, vv) / l).view(heads, d)
            lse[s, t] = (m + torch.log(l)).view(heads)
            # (a p that is nothing beside l may be off by any factor)
            w = (p / l) > 2.0 ** -40
            ep = torch.where(w, (d + 4) * U * mag + 6 * U * (x - m).abs() + 8 * U, 0.0).amax(dim=2, keepdim=True)
            cnt = x.shape[2]
            spread = torch.bmm(p, vv.abs()) / l
            to[s, t] = (2.0 ** -8 * o[s, t].view(c.kv, G, d).abs()
                        + (2 * ep + 2.0 ** -16 + 2 * cnt * U + 2.0 ** -20) * spread).view(heads, d)
            tl[s, t] = (ep[..., 0] + cnt * U + 2.0 ** -20).view(heads) + 2.0 ** -22 * lse[s, t].abs()
    return o, lse, to, tl


def attend(c, q, causal=False, scale=None, workspace=None, lse=True, stream=None):
    o = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device=q.device)
    ls = torch.full(q.shape[:3], float("nan"), dtype=torch.float32, device=q.device) if lse else None
    lc.lacache_paged_attention(q, c.k, c.v, c.table, c.lens, o, lse=ls, k_scale=c.k_scale, v_scale=c.v_scale,
                               scale=scale, causal=causal, workspace=workspace, stream=stream)
    return o, ls


def check_attention(c, q, causal, scale=None, what=""):
    o, lse = attend(c, q, causal, scale)
    ref, rl, to, tl = attention_exact(c, q, causal, scale)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(o).all()), what
    err = (o.double() - ref).abs()
    bad = err > to
    worst = float((err / to.clamp_min(1e-300)).nan_to_num(0.0).max())
    print("%s: max err %.3g, worst err/tolerance %.3f" % (what, float(err.max()), worst), flush=True)
    assert not bool(bad.any()), (what, worst)
    gone = rl == -math.inf
    assert torch.equal(lse == -math.inf, gone), what
    el = (lse.double() - rl).abs()[~gone]
    assert el.numel() == 0 or bool((el <= tl[~gone]).all()), (what, float((el / tl[~gone]).max()))
    return o, lse
