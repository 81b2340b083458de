"""The serving calls as a program runs them: prompts of odd lengths, their keys and values into pages, a fork, a compaction, and
tokens one by one and drafted, against one causal attention over everything that each sequence holds by then."""
import copy

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from serving_utils import check, f64, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sale():
    from paper_2505_24179_amd import sale as mod
    return mod


class _Sequence:
    """What one sequence has seen, on the host."""

    def __init__(self, k, v, pages):
        self.k, self.v, self.pages = k, v, list(pages)      # [Hkv, tokens, d]

    def add(self, k, v):
        self.k, self.v = np.concatenate([self.k, k], axis=1), np.concatenate([self.v, v], axis=1)


def _last(seqs, shared, q, n):
    """The oracle's results of the last n tokens of every sequence: its keys behind the shared ones."""
    got = []
    for s, seq in enumerate(seqs):
        k, v = np.concatenate([shared[0], seq.k], axis=1), np.concatenate([shared[1], seq.v], axis=1)
        total = k.shape[1]
        seen = np.arange(total)[None] <= (total - n + np.arange(n))[:, None]
        got.append([np.stack(x) for x in zip(*(so.attend(q[s, h], k[h // 2], v[h // 2], seen) for h in range(4)))])
    return [np.stack(x) for x in zip(*got)]


@pytest.mark.parametrize("page", [16, 64])
def test_a_program(sale, page):
    gen = torch.Generator().manual_seed(page)
    hq, hkv, n_pages = 4, 2, 64
    new = lambda n, h, b=1: rows((b, h, n, 128), "bnhd", gen)
    pools = [torch.full((n_pages, hkv, page, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    width = 8 if page == 64 else 24
    free = torch.randperm(n_pages, generator=gen).tolist()
    # a shared system prompt, computed and stored once
    prefix_len = 75
    pq, pk, pv = new(prefix_len, hq), new(prefix_len, hkv), new(prefix_len, hkv)
    p = sale.Params(1, hq, hkv, prefix_len)
    o, _ = sale.prompt_attn(p, pq, pk, pv)
    check(o, None, [x[None] for x in so.prompt(f64(pq)[0], f64(pk)[0], f64(pv)[0], [0, prefix_len])])
    prefix = [free.pop() for _ in range(-(-prefix_len // page))]
    table = torch.tensor([prefix + [-1] * (width - len(prefix))], dtype=torch.int32, device="cuda")
    sale.cache_append(p, sale.Cache(*pools, table, torch.tensor([prefix_len], dtype=torch.int32, device="cuda")), pk, pv)
    prefix = torch.tensor(prefix, dtype=torch.int32, device="cuda")
    shared = f64(pk)[0], f64(pv)[0]
    # three requests of odd lengths, one of them empty so far, packed into one call (here without the prefix before them)
    lens = [33, 0, 100]
    offsets = (0, 33, 33, 133)
    q, k, v = new(133, hq), new(133, hkv), new(133, hkv)
    p = sale.Params(1, hq, hkv, 133, cu_seqlens=offsets)
    o, _ = sale.prompt_attn(p, q, k, v)
    check(o, None, [x[None] for x in so.prompt(f64(q)[0], f64(k)[0], f64(v)[0], offsets)])
    seqs = [_Sequence(f64(k)[0, :, a:z], f64(v)[0, :, a:z], [free.pop() for _ in range(-(-max(1, z - a + 9) // page))])
            for a, z in zip(offsets[:-1], offsets[1:])]

    def cache():
        t = torch.full((len(seqs), width), -1, dtype=torch.int32)
        for s, seq in enumerate(seqs):
            t[s, :len(seq.pages)] = torch.tensor(seq.pages)
        held = torch.tensor([s.k.shape[1] for s in seqs], dtype=torch.int32)
        return sale.Cache(*pools, t.cuda(), held.cuda())

    sale.cache_append(p, cache(), k, v)

    def step(n):
        """n new tokens for every sequence: appended, then attended to."""
        kn, vn, qn = new(n, hkv, len(seqs)), new(n, hkv, len(seqs)), new(n, hq, len(seqs))
        for s, seq in enumerate(seqs):
            seq.add(f64(kn)[s], f64(vn)[s])
        ps, c = sale.Params(len(seqs), hq, hkv, n), cache()
        sale.cache_append(ps, c, kn, vn)
        got, lse = sale.decode_attn(ps, c, qn, prefix=prefix, prefix_len=prefix_len, want_lse=True)
        check(got, lse, _last(seqs, shared, f64(qn), n))

    step(1)
    step(3)
    # a fork of the third request: full pages are shared, the partly filled one is copied
    parent = seqs[2]
    full = parent.k.shape[1] // page
    fresh = [free.pop() for _ in parent.pages[full:]]
    c = cache()
    sale.cache_copy(sale.Params(1, hq, hkv, 1), c, parent.pages[full:], fresh)
    seqs.append(_Sequence(parent.k, parent.v, parent.pages[:full] + fresh))
    step(2)
    # the first request ends: its pages are spoiled, and everyone else's move to the lowest numbers that are free
    pools[0][seqs[0].pages] = float("nan")
    pools[1][seqs[0].pages] = float("nan")
    seqs = seqs[1:]
    used = sorted({x for s in seqs for x in s.pages} | set(prefix.tolist()))
    low = [x for x in range(len(used)) if x not in used]
    high = [x for x in used if x >= len(used)]
    sale.cache_copy(sale.Params(1, hq, hkv, 1), c, high, low)
    moved = dict(zip(high, low))
    for seq in seqs:
        seq.pages = [moved.get(x, x) for x in seq.pages]
    prefix = torch.tensor([moved.get(x, x) for x in prefix.tolist()], dtype=torch.int32, device="cuda")
    for pool in pools:
        pool[len(used):] = float("nan")
    step(1)


def test_caches_of_both_types_under_the_same_parameters(sale):
    """Sizes that are kept with the parameters are kept by the type of the pages, whose workspaces differ where there is much to read."""
    gen = torch.Generator().manual_seed(3)
    p, q = sale.Params(4, 8, 8, 1), rows((4, 8, 1, 128), "bhnd", gen)
    scale = torch.full((8,), 0.01, device="cuda")
    pages = torch.randn(40, 8, 16, 128, generator=gen).cuda()
    table = torch.full((4, 1024), -1, dtype=torch.int32)
    table[:, :10] = torch.arange(40, dtype=torch.int32).view(4, 10)
    table, lens = table.cuda(), torch.tensor([160, 3, 0, 77], dtype=torch.int32, device="cuda")
    bf16 = sale.Cache(pages.bfloat16(), pages.bfloat16(), table, lens)
    e4m3 = sale.Cache(*((pages / 0.01).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2)), table, lens, scale, scale)
    alone = [sale.decode_attn(sale.Params(4, 8, 8, 1), c, q)[0] for c in (bf16, e4m3)]
    assert sale.decode_workspace_bytes(p, bf16) != sale.decode_workspace_bytes(p, e4m3)
    for c, want in zip((bf16, e4m3), alone):
        assert torch.equal(sale.decode_attn(p, c, q)[0], want)


def test_copies_of_a_cache(sale):
    """A deep copy, made after calls, has pages, table and lens of its own; and pages whose tokens overlap are refused."""
    gen = torch.Generator().manual_seed(4)
    p = sale.Params(2, 4, 2, 1)
    pages = torch.randn(2, 4, 2, 16, 128, generator=gen).bfloat16().cuda()
    table = torch.tensor([[2, 0], [1, 3]], dtype=torch.int32, device="cuda")
    cache = sale.Cache(pages[0], pages[1], table, torch.tensor([20, 11], dtype=torch.int32, device="cuda"))
    q, new = rows((2, 4, 1, 128), "bhnd", gen), rows((2, 2, 1, 128), "bhnd", gen)
    before, _ = sale.decode_attn(p, cache, q)
    other = copy.deepcopy(cache)
    other.lens.add_(1)
    sale.cache_append(p, other, new, new)
    after, _ = sale.decode_attn(p, other, q)
    assert torch.equal(sale.decode_attn(p, cache, q)[0], before) and not torch.equal(after, before)
    flat = torch.zeros(128, dtype=torch.bfloat16, device="cuda").expand(1, 1, 16, 128)
    with pytest.raises(ValueError, match="apart"):
        sale.Cache(flat, flat, table, cache.lens)
