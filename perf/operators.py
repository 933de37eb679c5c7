"""Performance cases of the attention half of a layer that decodes over a paged
key/value cache, and of the 16-bit projections around it.

Three operators, used one after the other by a serving program:
  append  rotates the new tokens' queries and keys by their positions and
          stores keys and values in the pages of a cache
          (`lacache_paged_append`), bf16 or e4m3 with a scale per key;
  attn    the new tokens' attention over that cache
          (`lacache_paged_attention`): one token per sequence, or a block of
          them, grouped heads, sequences of different lengths;
  linear  act(a W^T + bias) + residual in bf16 (`lacache_linear_act_bf16`): the
          QKV projection with its bias, the output projection with the residual
          stream, the first layer's 16-bit gate/up product with its SwiGLU.

`own` chooses between the library's calls and the same operators in elementary
torch operations, in 32 bits and rounded once. Activations are N(0, s^2) with
1 % of the channels 40 times larger, s log-uniform in [0.5, 8], weights
N(0, 0.02^2), queries and keys N(0, 1.5^2), values N(0, 1); a sequence's pages
lie anywhere in the cache. Every input is drawn on the GPU from the seed.
"""

import math

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
BF16, FP8 = "bf16", "e4m3"
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh", "swiglu")


def listed():
    return [
        # one sequence decodes its next token: the smallest calls of a step
        _append("append_token1", 1, 1, 512, 32, 8, 128, 16, BF16),
        # 8 sequences write a 32-token block each (as many key as query heads) into an 8-bit cache
        _append("append_block8x32_e4m3", 8, 32, 1024, 32, 32, 128, 64, FP8),
        # prompts of 4 sequences, 2048 tokens each
        _append("append_prompt4x2048", 4, 2048, 2048, 32, 8, 128, 16, BF16),
        # the next token of one short sequence: latency
        _attn("attn_token1x500", 1, 1, 500, 500, 32, 8, 128, 16, BF16, True),
        # a batch of 48 sequences of very different lengths
        _attn("attn_tokens48_ragged", 48, 1, 1, 8191, 32, 8, 128, 16, BF16, True),
        # one sequence of 131072 tokens, 8-bit cache: the cache is split over its length
        _attn("attn_token1x131072_e4m3", 1, 1, 131072, 131072, 32, 8, 128, 64, FP8, True),
        # the denoising step of 8 sequences: a 32-token block sees all of its sequence, 32 heads
        _attn("attn_block8x32_1024", 8, 32, 700, 1024, 32, 32, 128, 64, BF16, False),
        # the largest: 64 sequences of up to 16384 tokens, 8-bit cache
        _attn("attn_tokens64x16384_e4m3", 64, 1, 12000, 16384, 64, 8, 128, 64, FP8, True),
        # the output projection of one 32-token block, added to the residual stream: the weights stream
        _linear("linear_out_block32", 32, 4096, 4096, "none", False, True),
        # the first layer's gate/up product with SwiGLU at the same rows
        _linear("linear_swiglu_block32", 32, 12288, 4096, "swiglu", False, False),
        # a short prompt of odd length through a biased layer with GELU
        _linear("linear_gelu_333", 333, 4096, 2048, "gelu", True, False),
        # 8 sequences of 1024 tokens: bias, SiLU and residual, bound by the products
        _linear("linear_silu_8192", 8192, 4096, 4096, "silu", True, True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choices(("append", "attn", "linear"), (2, 5, 3))[0]
    if kind == "linear":
        N, K = (max(128, log(128, 16384) // 128 * 128) for _ in range(2))
        act = rng.choice(ACTS)
        M = min(log(1, 8192), 8192 * 4096 * 4096 // (N * K * (2 if act == "swiglu" else 1)))
        return _linear(None, max(1, M), N, K, act, rng.random() < 0.5, rng.random() < 0.5)
    d = rng.choice((64, 128, 128))
    kv = rng.choice((1, 2, 4, 8, 8, 16, 32))
    heads = kv * rng.choice((1, 3, 4, 4, 7, 8))
    page = rng.choice((16, 16, 32, 64, 128, 256))
    cache = rng.choice((BF16, FP8))
    if kind == "append":
        nq = rng.choice((1, log(2, 64), log(64, 2048)))
        S = max(1, min(log(1, 256), 4 * 2048 * 48 * 128 // (nq * (heads + 2 * kv) * d)))
        return _append(None, S, nq, max(nq, log(64, 4096)), heads, kv, d, page, cache)
    nq = rng.choice((1, 1, log(2, 32)))
    longest = log(1, 131072)
    row = kv * d * (2 if cache == BF16 else 1)
    S = max(1, min(log(1, 256), 64 * 14000 * 8 * 128 // (longest * row), 2 ** 37 // (2 * d * heads * nq * longest)))
    return _attn(None, S, nq, rng.choice((1, longest)), longest, heads, kv, d, page, cache, rng.random() < 0.5)


def _named(name, case):
    return case if name is None else dict(case, name=name)


def _append(name, S, nq, longest, heads, kv, d, page, cache):
    """S sequences of up to `longest` tokens, the last nq of each appended."""
    return _named(name, {"kind": "append", "S": S, "nq": nq, "shortest": nq, "longest": longest, "heads": heads,
                         "kv": kv, "d": d, "page": page, "cache": cache})


def _attn(name, S, nq, shortest, longest, heads, kv, d, page, cache, causal):
    return _named(name, {"kind": "attn", "S": S, "nq": nq, "shortest": shortest, "longest": longest, "heads": heads,
                         "kv": kv, "d": d, "page": page, "cache": cache, "causal": causal})


def _linear(name, M, N, K, act, bias, residual):
    return _named(name, {"kind": "linear", "M": M, "N": N, "K": K, "act": act, "bias": bias, "residual": residual})


def _lengths(case):
    """The sequences' lengths: spread over [shortest, longest], in no order, the first the longest."""
    lo, hi, S = case["shortest"], case["longest"], case["S"]
    return [hi - (hi - lo) * ((i * 40503) % 65536) // 65536 for i in range(S)]


def _pages_of(case):
    return -(-case["longest"] // case["page"])


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) + 715339)


def _normal(g, shape, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std + mean).to(torch.bfloat16)


def _activations(g, M, H):
    s = 0.5 * 16.0 ** float(torch.rand((), generator=g, device=DEV))
    x = torch.randn((M, H), generator=g, device=DEV, dtype=torch.float32) * s
    wide = torch.randperm(H, generator=g, device=DEV)[: max(1, round(0.01 * H))]
    x[:, wide] *= 40.0
    return x.to(torch.bfloat16)


def _quantize(x):
    """Codes and scales of e4m3 with one scale per last axis: max|x| / 448."""
    s = x.abs().amax(dim=-1) / 448.0
    return (x / torch.where(s == 0, torch.ones_like(s), s)[..., None]).to(E4M3), s


def _cache(g, case, std):
    """Keys or values of every page, and their scales (None for bf16)."""
    shape = (case["S"] * _pages_of(case) + 3, case["kv"], case["page"], case["d"])
    x = _normal(g, shape, std)
    return (x, None) if case["cache"] == BF16 else _quantize(x.float())


def _table(g, case):
    """Every sequence's pages, anywhere in the cache."""
    S, mp = case["S"], _pages_of(case)
    return torch.randperm(S * mp + 3, generator=g, device=DEV)[: S * mp].view(S, mp).to(torch.int32)


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        rows = 2 * N if case["act"] == "swiglu" else N
        return {"a": _activations(g, M, K), "w": _normal(g, (rows, K), 0.02),
                "bias": _normal(g, (rows,), 0.5) if case["bias"] else None,
                "residual": _activations(g, M, N) if case["residual"] else None}
    S, nq, heads, kv, d = (case[k] for k in ("S", "nq", "heads", "kv", "d"))
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)
    s = {"table": _table(g, case)}
    s["k"], s["k_scale"] = _cache(g, case, 1.5)
    s["v"], s["v_scale"] = _cache(g, case, 1.0)
    if case["kind"] == "attn":
        s["lens"] = lens
        s["q"] = _normal(g, (S, nq, heads, d), 1.5)
        return s
    s["qkv"] = _normal(g, (S * nq, (heads + 2 * kv) * d), 1.5)
    s["seq"] = torch.arange(S, device=DEV, dtype=torch.int32).repeat_interleave(nq)
    s["pos"] = (lens[:, None] - nq + torch.arange(nq, device=DEV, dtype=torch.int32)).reshape(-1).contiguous()
    inv = 1.0 / 10000.0 ** (torch.arange(d // 2, device=DEV, dtype=torch.float64) / (d // 2))
    ang = torch.arange(case["longest"], device=DEV, dtype=torch.float64)[:, None] * inv[None, :]
    s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    if case["kind"] == "linear":
        s["out"] = torch.empty((case["M"], case["N"]), dtype=torch.bfloat16, device=DEV)
    elif case["kind"] == "attn":
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], dtype=torch.float32, device=DEV)
    else:
        s["q"] = torch.empty((case["S"] * case["nq"], case["heads"], case["d"]), dtype=torch.bfloat16, device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"append": _own_append, "attn": _own_attn, "linear": _own_linear}[kind](state)
    return {"append": _plain_append, "attn": _plain_attn, "linear": _plain_linear}[kind](state)


def _written(s):
    """What an append leaves: the rotated queries and the caches."""
    return [s["q"], s["k"], s["v"]] + ([] if s["k_scale"] is None else [s["k_scale"], s["v_scale"]])


def _own_append(s):
    import paper_2607_16339_amd as lc

    lc.lacache_paged_append(s["qkv"], s["seq"], s["pos"], s["cos"], s["sin"], s["table"], s["q"], s["k"], s["v"],
                            s["k_scale"], s["v_scale"])
    return _written(s)


def _own_attn(s):
    import paper_2607_16339_amd as lc

    lc.lacache_paged_attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["o"], lse=s["lse"],
                               k_scale=s["k_scale"], v_scale=s["v_scale"], causal=s["case"]["causal"])
    return [s["o"], s["lse"]]


def _own_linear(s):
    import paper_2607_16339_amd as lc

    lc.lacache_linear_act_bf16(s["a"], s["w"], s["out"], bias=s["bias"], residual=s["residual"],
                               act=ACTS.index(s["case"]["act"]))
    return [s["out"]]


def _rotate(x, cos, sin):
    """x [T, heads, d] in fp32, cos and sin [T, 1, d / 2]."""
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _plain_append(s):
    case = s["case"]
    heads, kv, d, page = case["heads"], case["kv"], case["d"], case["page"]
    x = s["qkv"].view(-1, heads + 2 * kv, d).float()
    pos, seq = s["pos"].long(), s["seq"].long()
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    s["q"].copy_(_rotate(x[:, :heads], cos, sin))
    at, slot = s["table"][seq, pos // page].long(), pos % page
    for_cache = ((s["k"], s["k_scale"], _rotate(x[:, heads:heads + kv], cos, sin)),
                 (s["v"], s["v_scale"], x[:, heads + kv:]))
    _store(at, slot, *for_cache[0])
    _store(at, slot, *for_cache[1])
    return _written(s)


def _store(at, slot, cache, scale, x):
    if scale is None:
        cache[at, :, slot] = x.to(torch.bfloat16)
    else:
        codes, s = _quantize(x)
        cache.view(torch.uint8)[at, :, slot] = codes.view(torch.uint8)
        scale[at, :, slot] = s


def _gathered(cache, scale, table):
    """[S, kv, keys, d] in fp32."""
    at = table.long()
    x = cache.view(torch.uint8)[at].view(E4M3).float() * scale[at][..., None] if scale is not None else cache[at].float()
    S, mp, kv, page, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(S, kv, mp * page, d)


def _plain_attn(s):
    case = s["case"]
    S, nq, heads, kv, d = (case[k] for k in ("S", "nq", "heads", "kv", "d"))
    k, v = _gathered(s["k"], s["k_scale"], s["table"]), _gathered(s["v"], s["v_scale"], s["table"])
    q = s["q"].float().view(S, nq, kv, heads // kv, d).permute(0, 2, 1, 3, 4).reshape(S, kv, -1, d)
    score = torch.matmul(q, k.transpose(2, 3)).view(S, kv, nq, heads // kv, -1) * (1.0 / math.sqrt(d))
    end = s["lens"].long()[:, None].expand(S, nq)
    if case["causal"]:
        end = end - nq + 1 + torch.arange(nq, device=q.device)
    seen = torch.arange(k.shape[2], device=q.device) < end[:, :, None]  # [S, nq, keys]
    score = torch.where(seen[:, None, :, None], score, torch.full_like(score, -math.inf))
    top = score.amax(dim=-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(S, kv, -1, p.shape[-1]), v).view(S, kv, nq, heads // kv, d)
    o = torch.where(total == 0, torch.zeros_like(o), o / total)
    s["o"].copy_(o.permute(0, 2, 1, 3, 4).reshape(S, nq, heads, d))
    s["lse"].copy_((top + torch.log(total))[..., 0].permute(0, 2, 1, 3).reshape(S, nq, heads))
    return [s["o"], s["lse"]]


def _act(name, x):
    if name == "relu":
        return torch.where(x < 0, torch.zeros_like(x), x)
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _plain_linear(s):
    act = s["case"]["act"]
    y = torch.matmul(s["a"].float(), s["w"].float().t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if act == "swiglu":
        g, u = y.chunk(2, dim=1)
        y = _act("silu", g) * u
    else:
        y = _act(act, y)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    s["out"].copy_(y)
    return [s["out"]]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        rows = 2 * N if case["act"] == "swiglu" else N
        extra = (2 * rows if case["bias"] else 0) + (2 * M * N if case["residual"] else 0)
        return {"bytes": 2 * (M * K + rows * K + M * N) + extra, "flops": 2 * M * rows * K}
    S, nq, heads, kv, d, page = (case[k] for k in ("S", "nq", "heads", "kv", "d", "page"))
    key = kv * (4 * d if case["cache"] == BF16 else 2 * d + 8)  # a key and a value of every head
    lens = _lengths(case)
    if case["kind"] == "append":
        T = S * nq
        pages = sum(-(-n // page) - (n - nq) // page for n in lens)
        positions = min(T, case["longest"])
        return {"bytes": T * (2 * (heads + 2 * kv) * d + 2 * heads * d + key + 8) + 4 * pages + 4 * d * positions,
                "flops": 3 * T * (heads + kv) * d}
    pages = sum(-(-n // page) for n in lens)
    pairs = sum(max(0, n - nq + t + 1) if case["causal"] else n for n in lens for t in range(nq))
    return {"bytes": sum(lens) * key + 4 * pages + 4 * S + S * nq * heads * (4 * d + 4), "flops": 4 * d * heads * pairs}


# ---------------------------------------------------------------------------
# the same outputs in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "linear": _exact_linear}[case["kind"]](case, s)


def _exact_append(case, s):
    heads, kv, d, page = case["heads"], case["kv"], case["d"], case["page"]
    T, h = case["S"] * case["nq"], d // 2
    x = s["qkv"].double().view(T, heads + 2 * kv, d)
    c, n = s["cos"].double()[s["pos"].long()], s["sin"].double()[s["pos"].long()]
    turned = torch.empty((T, heads + kv, d), dtype=torch.float64, device=DEV)
    turned[..., :h] = x[:, :heads + kv, :h] * c[:, None] - x[:, :heads + kv, h:] * n[:, None]
    turned[..., h:] = x[:, :heads + kv, h:] * c[:, None] + x[:, :heads + kv, :h] * n[:, None]
    row = s["table"][s["seq"].long(), (s["pos"] // page).long()].long() * page + (s["pos"] % page).long()
    out, scales = [turned[:, :heads]], []
    for name, new in (("k", turned[:, heads:]), ("v", x[:, heads + kv:])):
        cache = s[name].double().permute(0, 2, 1, 3).reshape(-1, kv, d)  # a row per place in the cache
        if s[name + "_scale"] is None:
            cache[row] = new
        else:
            top = new.abs().amax(dim=2) / 448.0
            cache[row] = new / top[..., None]  # a code stands for its value in units of the scale
            scale = s[name + "_scale"].double().permute(0, 2, 1).reshape(-1, kv)
            scale[row] = top
            scales.append(scale.view(-1, page, kv).permute(0, 2, 1))
        out.append(cache.view(-1, page, kv, d).permute(0, 2, 1, 3))
    return out + scales


def _exact_attn(case, s):
    S, nq, heads, kv, d, page = (case[k] for k in ("S", "nq", "heads", "kv", "d", "page"))
    o = torch.zeros((S, nq, heads, d), dtype=torch.float64, device=DEV)
    lse = torch.full((S, nq, heads), -math.inf, dtype=torch.float64, device=DEV)
    for i, n in enumerate(_lengths(case)):
        at = s["table"][i, : -(-n // page)].long()
        kd, vd = s["k"].view(torch.uint8)[at].view(s["k"].dtype).double(), None
        vd = s["v"].view(torch.uint8)[at].view(s["v"].dtype).double()
        if s["k_scale"] is not None:
            kd, vd = kd * s["k_scale"][at].double()[..., None], vd * s["v_scale"][at].double()[..., None]
        kd, vd = (t.transpose(0, 1).reshape(kv, -1, d)[:, :n] for t in (kd, vd))
        # tokens 0 .. skip - 1 come before the sequence's first key
        skip = max(0, nq - n) if case["causal"] else 0
        rows = nq - skip
        qd = s["q"][i, skip:].double().view(rows, kv, heads // kv, d).transpose(0, 1).reshape(kv, -1, d)
        score = torch.bmm(qd, kd.transpose(1, 2).contiguous()).view(kv, rows, heads // kv, n) / math.sqrt(d)
        if case["causal"]:
            ahead = torch.ones((rows, n), dtype=torch.bool, device=DEV).triu(n - rows + 1)
            score.masked_fill_(ahead[None, :, None], -math.inf)
        lse[i, skip:] = torch.logsumexp(score, dim=3).transpose(0, 1).reshape(rows, heads)
        p = torch.softmax(score, dim=3).view(kv, -1, n)
        o[i, skip:] = torch.bmm(p, vd.contiguous()).view(kv, rows, heads // kv, d).transpose(0, 1).reshape(rows, heads, d)
    return [o, lse]


def _exact_linear(case, s):
    N = case["N"]
    y = s["a"].double() @ s["w"].double().t().contiguous()
    if s["bias"] is not None:
        y += s["bias"].double()
    act = case["act"]
    if act == "relu":
        y = y.clamp_min(0.0)
    elif act == "silu":
        y = y * torch.sigmoid(y)
    elif act == "gelu":
        y = y * 0.5 * torch.erfc(-y / math.sqrt(2.0))
    elif act == "gelu_tanh":
        y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
    elif act == "swiglu":
        y = y[:, :N] * torch.sigmoid(y[:, :N]) * y[:, N:]
    return [y if s["residual"] is None else y + s["residual"].double()]
