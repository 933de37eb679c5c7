"""That no key is lost or taken twice where a sequence is cut: into tiles, into
wavefronts' runs, into pieces and their shares of the join.

Queries of zeros give every key the same weight, so l is the number of keys,
exactly, and lse its logarithm: one key of 100000 more or less moves it by 1e-5,
a hundred times its rounding. Values are 1 in one dimension per key and 0
elsewhere, so o times the number of keys counts the keys of each dimension, at
most 104 of them: one more or less is 2.4 times the rounding of o (2^-8). Two
patterns together tell any two keys of up to d^2 apart."""

import math

import pytest
import torch

from paged_util import DEV, Cache, attend, check_attention, normal, quantize

pytestmark = pytest.mark.gpu

# nq, heads, kv, sequences. Rows per KV head: 4 and 16 (8 wavefronts that split the keys; 4 of them
# where the sequences fill the chip), 40, 64 (two row tiles of 16), 80, 208, 384 (wavefronts that split the rows)
FORMS = [(1, 8, 2, 7), (4, 4, 1, 7), (1, 16, 16, 40), (1, 256, 16, 40), (5, 8, 1, 7), (16, 64, 16, 40), (40, 2, 1, 7),
         (26, 16, 2, 7), (64, 6, 1, 3), (5, 256, 16, 9), (1, 1, 1, 140)]


def _lengths(S, d):
    """Up to 104 keys per dimension, around borders of tiles and of pieces, then short ones."""
    lens = [104 * d - 1, 64 * d + 1, 33 * d, 32 * d + 1, 8 * d + 1, 0, 517][:S]
    return lens + [(61 * i) % 300 for i in range(S - len(lens))]


def _mark(c, lens, pattern):
    """Values: 1 in dimension pattern(key) + head (none where that is negative)."""
    byte = c.v.view(torch.uint8)
    for s, n in enumerate(lens):
        if n == 0:
            continue
        j = torch.arange(n)
        page, slot = c.table[s].cpu().long()[j // c.page], j % c.page
        for h in range(c.kv):
            dim = pattern(j)
            x = torch.zeros((n, c.d))
            x[j[dim >= 0], ((dim + h) % c.d)[dim >= 0]] = 1.0
            if c.fp8:
                byte[page.to(DEV), h, slot.to(DEV)] = (x * 0x38).to(torch.uint8).to(DEV)  # 0x38: 1.0
                c.v_scale[page.to(DEV), h, slot.to(DEV)] = 1.0
            else:
                c.v[page.to(DEV), h, slot.to(DEV)] = x.to(torch.bfloat16).to(DEV)


def _count(c, lens, pattern, nq, causal):
    """(keys of each dimension [S, nq, kv, d], keys [S, nq]) that the rows see."""
    S = len(lens)
    count, keys = torch.zeros((S, nq, c.kv, c.d), dtype=torch.float64), torch.zeros((S, nq), dtype=torch.float64)
    for s, n in enumerate(lens):
        dim = pattern(torch.arange(n))
        for t in range(nq):
            m = max(0, n - nq + t + 1) if causal else n
            seen = dim[:m]
            b = torch.bincount(seen[seen >= 0] % c.d, minlength=c.d).double()
            keys[s, t] = m
            for h in range(c.kv):
                count[s, t, h] = b.roll(h)
    return count, keys


def _check(c, lens, patterns, nq, causal, most=104):
    q = torch.zeros((c.S, nq, c.heads, c.d), dtype=torch.bfloat16, device=DEV)
    for k, pattern in enumerate(patterns):
        _mark(c, lens, pattern)
        count, keys = _count(c, lens, pattern, nq, causal)
        assert float(count.max()) <= most
        o, lse = attend(c, q, causal)
        torch.cuda.synchronize()
        lse, o = lse.cpu().double(), o.cpu().double().view(c.S, nq, c.kv, -1, c.d)
        want = torch.log(keys)[:, :, None].expand_as(lse)
        none = keys[:, :, None].expand_as(lse) == 0
        assert torch.equal(lse == -math.inf, none)
        # (log2 of a whole number, its product with ln 2 and the hardware's logarithm: 4 roundings of the value)
        assert bool(((lse - want).abs()[~none] <= 2.0 ** -22 * want[~none] + 1e-12).all()), k
        ref = count / keys.clamp_min(1.0)[:, :, None, None]
        assert bool(((o - ref[:, :, :, None]).abs() <= (2.0 ** -8 + 2.0 ** -21) * ref[:, :, :, None]).all()), k


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,heads,kv,S", FORMS)
def test_every_key_counts_once(nq, heads, kv, S, d, fp8, causal):
    lens = _lengths(S, d)
    c = Cache(lens, heads, kv, d, 16 if d == 64 else 64, fp8, seed=nq + heads)
    run = 104 if d == 128 else 52  # (shorter than d)
    _check(c, lens, (lambda j: j % d, lambda j: (j // run) % d), nq, causal)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("nq,heads,kv", [(1, 8, 2), (4, 4, 1), (5, 8, 1), (12, 8, 1)])
def test_every_key_counts_once_in_a_long_sequence(nq, heads, kv, fp8):
    """The keys on both sides of every 32nd key's border, of more pieces than a join's shares hold at once."""
    lens = [100001, 40]
    c = Cache(lens, heads, kv, 128, 256, fp8, seed=nq)
    border = lambda j: torch.where(j % 32 == 0, j // 16, torch.where(j % 32 == 31, j // 16, torch.full_like(j, -1)))  # noqa: E731
    _check(c, lens, (border,), nq, True)


def _q(c, nq, seed=1, std=1.5):
    return normal(torch.Generator().manual_seed(seed), (c.S, nq, c.heads, c.d), std).to(DEV)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,heads,kv", [(40, 2, 1), (26, 16, 2)])
def test_bad_pages_where_wavefronts_split_the_rows(nq, heads, kv, d, fp8, causal):
    """Keys on pages of no number are left out, in whole sequences and in cut ones."""
    c = Cache([300, 200, 100, 64, 2000], heads, kv, d, 16, fp8, seed=11)
    c.table[0, 3], c.table[0, 7], c.table[1, 0] = -1, c.num_pages, 2 ** 31 - 1
    c.table[2] = -1  # no key at all
    c.lens[3] = -5
    c.table[4, 30:40], c.table[4, 77] = -2 ** 31, c.num_pages + 5
    o, lse = check_attention(c, _q(c, nq), causal, what="bad pages")
    assert bool((o[2] == 0).all()) and bool((lse[2] == -math.inf).all()) and bool((o[3] == 0).all())


@pytest.mark.parametrize("step", [0.3, 0.1, 0.02, -0.1])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,heads,kv", [(2, 4, 1), (20, 2, 1), (40, 2, 1), (26, 16, 2)])
def test_scores_that_climb_through_the_keys(nq, heads, kv, d, fp8, step):
    """Scores that grow by `step` (in powers of 2) from key to key, by several times or a part of
    the 8 by which a base may lag in every tile, or that fall; noise of one power beside it."""
    lens = [700, 1500, 33]
    c = Cache(lens, heads, kv, d, 16, fp8, seed=29, kstd=0.0)
    g = torch.Generator().manual_seed(30)
    for s, n in enumerate(lens):
        j = torch.arange(n)
        page, slot = c.table[s].cpu().long()[j // 16].to(DEV), (j % 16).to(DEV)
        climb = step * j * math.log(2.0) / math.sqrt(d)  # of each of the d dims, for a query of ones
        for h in range(kv):
            k = (climb[:, None] + torch.randn((n, d), generator=g) * math.log(2.0)).to(torch.bfloat16)
            if fp8:
                codes, scale = quantize(k.float())
                c.k.view(torch.uint8)[page, h, slot] = codes.view(torch.uint8).to(DEV)
                c.k_scale[page, h, slot] = scale.to(DEV)
            else:
                c.k[page, h, slot] = k.to(DEV)
    q = (1.0 + 0.1 * torch.randn((c.S, nq, heads, d), generator=g)).to(torch.bfloat16).to(DEV)
    check_attention(c, q, True, scale=1.0 / math.sqrt(d), what="step %g" % step)
