"""decode_attn against the oracle: heads, new tokens, page sizes and types, layouts, lengths from none, prefixes, and everything
that is in the place of a key and is none.  Whatever is no key holds NaN here."""
import numpy as np
import pytest
import torch

from serving_utils import bits, check, decode_oracle, f64, make_cache, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sale():
    from paper_2505_24179_amd import sale as mod
    return mod


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 130, 517]


@pytest.mark.parametrize("hq,hkv,n,page,kind,layout,prefix_len", [
    (4, 4, 1, 16, "bf16", "bhnd", 0), (4, 4, 1, 16, "bf16", "bnhd", 1), (6, 2, 1, 32, "bf16", "padded", 0), (6, 2, 3, 16, "fp8", "bnhd", 16),
    (8, 2, 1, 64, "fp8", "bhnd", 0), (8, 2, 4, 64, "bf16", "bhnd", 31), (8, 2, 7, 128, "bf16", "bnhd", 33), (8, 1, 8, 256, "fp8", "padded", 300),
    (16, 1, 1, 16, "bf16", "bhnd", 129), (34, 2, 1, 32, "fp8", "bhnd", 40), (64, 1, 1, 32, "bf16", "bhnd", 47), (5, 1, 12, 16, "bf16", "padded", 260),
    (1, 1, 64, 64, "bf16", "bhnd", 20), (1, 1, 1, 16, "fp8", "bhnd", 15)])
def test_against_the_oracle(sale, hq, hkv, n, page, kind, layout, prefix_len):
    gen = torch.Generator().manual_seed(hq * 1000 + n * 10 + page)
    cache, prefix = make_cache(sale, LENS, hkv, page, kind, layout, gen, prefix_len)
    p = sale.Params(len(LENS), hq, hkv, n)
    q = rows((len(LENS), hq, n, 128), layout, gen, 2.0)
    o, lse = sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    check(o, lse, decode_oracle(cache, q, prefix, prefix_len))
    again, _ = sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=prefix_len)
    assert torch.equal(bits(again), bits(o))      # no order of anything enters the result


@pytest.mark.parametrize("batch,longest,prefix_len,kind", [(1, 5000, 0, "bf16"), (2, 9001, 4100, "bf16"), (40, 700, 0, "fp8"), (70, 300, 2049, "bf16"),
                                                           (300, 40, 100, "fp8")])
def test_many_parts_and_many_rows(sale, batch, longest, prefix_len, kind):
    """Long sequences cut over many workgroups, and batches whose rows fill several tiles of the prefix; a sample of the rows."""
    gen = torch.Generator().manual_seed(batch + longest)
    lens = [longest] + [int(x) for x in torch.randint(0, longest, (batch - 1,), generator=gen)]
    cache, prefix = make_cache(sale, lens, 2, 16, kind, "bhnd", gen, prefix_len, spoil=False)
    q = rows((batch, 8, 1, 128), "bhnd", gen, 2.0)
    o, lse = sale.decode_attn(sale.Params(batch, 8, 2, 1), cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    some = sorted({0, batch // 3, batch - 1})
    part = sale.Cache(cache.k, cache.v, cache.table[some].contiguous(), cache.lens[some].contiguous(), cache.k_scale, cache.v_scale)
    check(o[some], lse[some], decode_oracle(part, q[some], prefix, prefix_len))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("n", [5, 12])
@pytest.mark.parametrize("page", [16, 128])
def test_more_rows_than_a_tile_and_long_sequences(sale, kind, n, page):
    gen = torch.Generator().manual_seed(n + page)
    cache, prefix = make_cache(sale, [3000, 7, 1100, 0, 2049], 1, page, kind, "bnhd", gen, 0)
    q = rows((5, 4, n, 128), "bnhd", gen, 2.0)
    o, lse = sale.decode_attn(sale.Params(5, 4, 1, n), cache, q, want_lse=True)
    check(o, lse, decode_oracle(cache, q, None, 0))


def _some(sale, cache, q, o, lse, prefix, prefix_len, some):
    part = sale.Cache(cache.k, cache.v, cache.table[some].contiguous(), cache.lens[some].contiguous(), cache.k_scale, cache.v_scale)
    check(o[some], lse[some], decode_oracle(part, q[some], prefix, prefix_len))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("page,layout", [(16, "bhnd"), (32, "bnhd"), (64, "padded")])
@pytest.mark.parametrize("batch,n,prefix_len", [(9, 2, 12000), (40, 1, 7001), (33, 3, 4133)])
def test_many_rows_and_a_long_prefix(sale, kind, page, layout, batch, n, prefix_len):
    """64 rows and more against many steps of the prefix, of whole pages and of what is left."""
    gen = torch.Generator().manual_seed(batch + page)
    cache, prefix = make_cache(sale, [3 + s % 5 for s in range(batch)], 1, page, kind, layout, gen, prefix_len)
    q = rows((batch, 4, n, 128), layout, gen, 2.0)
    o, lse = sale.decode_attn(sale.Params(batch, 4, 1, n), cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    _some(sale, cache, q, o, lse, prefix, prefix_len, [0, batch // 2, batch - 1])
    again, _ = sale.decode_attn(sale.Params(batch, 4, 1, n), cache, q, prefix=prefix, prefix_len=prefix_len)
    assert torch.equal(bits(again), bits(o))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("how", ["rising", "falling", "late", "huge", "missing"])
def test_scores_of_a_long_prefix(sale, kind, page, how):
    """Maxima that rise in every step, or in the first or last ones alone; scores of some ten thousands; pages that are none."""
    gen = torch.Generator().manual_seed(page)
    batch, prefix_len = 40, 5000
    cache, prefix = make_cache(sale, [4] * batch, 1, page, kind, "bhnd", gen, prefix_len, spoil=False)
    n_prefix = len(prefix)
    ramp = {"rising": torch.linspace(0.01, 4, n_prefix), "falling": torch.linspace(4, 0.01, n_prefix), "late": torch.cat([torch.full((n_prefix - 1,), 0.01), torch.ones(1) * 4]),
            "huge": torch.linspace(1, 60, n_prefix), "missing": torch.ones(n_prefix)}[how].cuda()
    at = prefix.long()
    if kind == "bf16":
        cache.k[at] = (cache.k[at].float() * ramp[:, None, None, None]).bfloat16()
    else:
        codes = (cache.k.float() * 0.1)
        codes[at] *= ramp[:, None, None, None]
        cache.k.copy_(codes.clamp(-448, 448).to(torch.float8_e4m3fn))
        cache.k_scale.mul_(10.0)
    if how == "missing":
        prefix[n_prefix // 2], prefix[n_prefix - 1], prefix[3] = -1, cache.k.shape[0], 2 ** 31 - 1
    q = rows((batch, 4, 1, 128), "bhnd", gen, 3.0)
    o, lse = sale.decode_attn(sale.Params(batch, 4, 1, 1), cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    _some(sale, cache, q, o, lse, prefix, prefix_len, [0, 17, batch - 1])


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_pages_that_are_none_and_lens_that_lie(sale, kind):
    gen = torch.Generator().manual_seed(7)
    cache, prefix = make_cache(sale, [100, 100, 100, 64, 40, 70], 2, 16, kind, "bhnd", gen, 50, room=0, spoil=False)
    cache.table[0, 2], cache.table[0, 6] = -1, cache.k.shape[0]
    cache.table[1, :] = 2 ** 31 - 1
    cache.table[2, 0], cache.table[2, 1] = -2 ** 31, cache.k.shape[0] + 5
    cache.lens[3], cache.lens[4], cache.lens[5] = 2 ** 31 - 1, -7, 113       # beyond the table, negative, one token beyond the table
    prefix[1] = -3
    q = rows((6, 8, 2, 128), "bhnd", gen, 2.0)
    for pre in (50, 0):
        o, lse = sale.decode_attn(sale.Params(6, 8, 2, 2), cache, q, prefix=prefix, prefix_len=pre, want_lse=True)
        check(o, lse, decode_oracle(cache, q, prefix, pre))


@pytest.mark.parametrize("kind,page,value", [("bf16", 16, "nan"), ("bf16", 16, "inf"), ("fp8", 64, "nan")])      # (E4M3 has no infinity)
def test_a_new_token_does_not_reach_those_before_it(sale, kind, page, value):
    gen = torch.Generator().manual_seed(8)
    lens, n = [40, 65, 5, 32], 4
    cache, prefix = make_cache(sale, lens, 2, page, kind, "bhnd", gen, 20)
    for s, back in ((0, 1), (1, 2), (2, 3), (3, 1)):      # the last token, the one before, ...
        pos = lens[s] - back
        at = (int(cache.table[s, pos // page]), slice(None), pos % page)
        if s % 2 == 0:
            bits(cache.k)[at] = bits(torch.tensor(float(value)).to(cache.k.dtype).cuda())
        bits(cache.v)[at + (slice(0, 128, 3),)] = bits(torch.tensor(float(value)).to(cache.v.dtype).cuda())
    q = rows((4, 6, n, 128), "bhnd", gen)
    o, lse = sale.decode_attn(sale.Params(4, 6, 2, n), cache, q, prefix=prefix, prefix_len=20, want_lse=True)
    want = decode_oracle(cache, q, prefix, 20)
    for s, back in ((0, 1), (1, 2), (2, 3), (3, 1)):
        sound = slice(0, n - back)
        assert torch.isfinite(o[s, :, sound]).all()
        check(o[s:s + 1, :, sound], lse[s:s + 1, :, sound], [x[s:s + 1, :, sound] for x in want])
        if value == "nan":
            assert torch.isnan(o[s, :, n - back:, 0:128:3]).all()


@pytest.mark.parametrize("hq,prefix_len", [(4, 0), (4, 40), (24, 0), (40, 200)])
def test_infinite_values_that_are_seen(sale, hq, prefix_len):
    """An infinity in V is one in O, of its sign, whatever the probability's last bits are; one of each sign is NaN."""
    gen = torch.Generator().manual_seed(16)
    cache, prefix = make_cache(sale, [70, 45, 130], 1, 16, "bf16", "bhnd", gen, prefix_len, spoil=False)
    v = cache.v
    v[int(cache.table[0, 1]), 0, 3, 7], v[int(cache.table[0, 1]), 0, 4, 8] = float("inf"), -float("inf")
    v[int(cache.table[1, 0]), 0, 5, 9] = v[int(cache.table[1, 2]), 0, 2, 9] = float("inf")
    v[int(cache.table[2, 0]), 0, 5, 9], v[int(cache.table[2, 7]), 0, 0, 9] = float("inf"), -float("inf")
    q = rows((3, hq, 1, 128), "bhnd", gen, 0.5)
    q[0] = 0      # (all probabilities equal)
    o, lse = sale.decode_attn(sale.Params(3, hq, 1, 1), cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    check(o, lse, decode_oracle(cache, q, prefix, prefix_len))
    assert bool((o[0, :, 0, 7] == float("inf")).all() and (o[0, :, 0, 8] == -float("inf")).all() and torch.isnan(o[2, :, 0, 9]).all())


def test_a_query_that_is_not_finite_stays_alone(sale):
    gen = torch.Generator().manual_seed(9)
    cache, prefix = make_cache(sale, [50, 60, 70], 1, 16, "bf16", "bhnd", gen, 40)
    q = rows((3, 4, 2, 128), "bhnd", gen)
    clean, _ = sale.decode_attn(sale.Params(3, 4, 1, 2), cache, q, prefix=prefix, prefix_len=40)
    q[1, 2, 0, 5] = float("nan")
    q[2, 0, 1, 9] = float("inf")
    o, _ = sale.decode_attn(sale.Params(3, 4, 1, 2), cache, q, prefix=prefix, prefix_len=40)
    assert torch.isnan(o[1, 2, 0]).all() and torch.isnan(o[2, 0, 1]).all()
    hit = torch.zeros(3, 4, 2, dtype=torch.bool, device="cuda")
    hit[1, 2, 0] = hit[2, 0, 1] = True
    assert torch.equal(o[~hit], clean[~hit])


def test_large_values_and_scores(sale):
    """V near the largest bf16, scores of some thousands with a maximum that rises late, equal scores."""
    gen = torch.Generator().manual_seed(10)
    cache, _ = make_cache(sale, [700, 700, 700], 1, 16, "bf16", "bhnd", gen, spoil=False)
    n_pages = cache.k.shape[0]
    cache.v.mul_(0).add_(3.2e38)
    cache.k.mul_(torch.linspace(0.1, 60.0, n_pages, device="cuda")[:, None, None, None].bfloat16())
    q = rows((3, 4, 1, 128), "bhnd", gen, 3.0)
    q[1] *= 1e-30
    o, lse = sale.decode_attn(sale.Params(3, 4, 1, 1), cache, q, want_lse=True)
    check(o, lse, decode_oracle(cache, q, None, 0))
    assert torch.isfinite(o).all()


def test_nothing_beyond_the_outputs_is_written(sale):
    gen = torch.Generator().manual_seed(11)
    cache, prefix = make_cache(sale, [33, 0, 90], 2, 16, "bf16", "bhnd", gen, 35)
    p = sale.Params(3, 6, 2, 3)
    q = rows((3, 6, 3, 128), "bhnd", gen)
    plain, _ = sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=35)
    before = bits(cache.k).clone(), bits(cache.v).clone()
    big = torch.full((4, 8, 5, 160), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[:3, 1:7, 1:4, 16:144]
    need = sale.decode_workspace_bytes(p, cache, 35)
    ws = torch.full((need + 4096,), 173, dtype=torch.uint8, device="cuda")
    sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=35, out=out, ws=ws[:need])
    assert torch.equal(out, plain) and bool((ws[need:] == 173).all())
    out.fill_(7.0)
    assert bool((big == 7.0).all())
    assert torch.equal(bits(cache.k), before[0]) and torch.equal(bits(cache.v), before[1])


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_offsets_beyond_32_bits(sale, kind):
    """Pages at the far end of pools of more than 4 GB each."""
    gen = torch.Generator().manual_seed(12)
    size = 2 if kind == "bf16" else 1
    n_pages = (5 << 30) // (128 * 128 * 8 * size)
    small, _ = make_cache(sale, [300], 8, 128, kind, "bhnd", gen, spoil=False)
    far = [n_pages - 1, 3, n_pages - 4]
    k = torch.empty(n_pages, 8, 128, 128, dtype=torch.uint8 if size == 1 else torch.int16, device="cuda")
    v = torch.empty_like(k)
    for i, at in enumerate(far):
        k[at], v[at] = bits(small.k)[int(small.table[0, i])], bits(small.v)[int(small.table[0, i])]
    big = sale.Cache(k.view(small.k.dtype), v.view(small.v.dtype), torch.tensor([far], dtype=torch.int32, device="cuda"), small.lens,
                     small.k_scale, small.v_scale)
    q = rows((1, 8, 1, 128), "bhnd", gen)
    near = sale.Cache(small.k, small.v, small.table[:, :3].contiguous(), small.lens, small.k_scale, small.v_scale)
    p = sale.Params(1, 8, 8, 1)
    assert torch.equal(sale.decode_attn(p, big, q)[0], sale.decode_attn(p, near, q)[0])


def test_captured_with_lens_that_grow(sale):
    """Captured once; lens, table, queries and pages change between the replays.  Two graphs with workspaces of their own."""
    gen = torch.Generator().manual_seed(13)
    lens = [0, 17, 60, 250]
    cache, prefix = make_cache(sale, lens, 2, 16, "bf16", "bhnd", gen, 77, room=3, spoil=False)
    p = sale.Params(4, 8, 2, 1)
    q, new = rows((4, 8, 1, 128), "bhnd", gen), rows((4, 2, 1, 128), "bhnd", gen)
    free = [i for i in range(cache.k.shape[0]) if i not in set(cache.table.flatten().tolist()) | set(prefix.tolist())]
    cache.table[0, 0], cache.table[2, 4] = free[0], free[1]      # (room for the tokens to come)
    o = torch.empty_like(q)
    ws = torch.empty(sale.decode_workspace_bytes(p, cache, 77), dtype=torch.uint8, device="cuda")

    def step():
        cache.lens.add_(1)
        sale.cache_append(p, cache, new, new)
        sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=77, out=o, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        cache.lens.sub_(1)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for replay in range(5):
        q.copy_(rows((4, 8, 1, 128), "bhnd", gen))
        new.copy_(rows((4, 2, 1, 128), "bhnd", gen))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert cache.lens.tolist() == [n + 1 + replay for n in lens]
        eager, _ = sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=77)
        assert torch.equal(eager, o)
        for s in range(4):
            pos = lens[s] + replay
            page = int(cache.table[s, pos // 16])
            assert torch.equal(cache.k[page, :, pos % 16], new[s, :, 0])


def test_on_another_stream(sale):
    gen = torch.Generator().manual_seed(14)
    cache, prefix = make_cache(sale, [900, 20], 2, 32, "bf16", "bhnd", gen, 64, spoil=False)
    p, q = sale.Params(2, 8, 2, 1), rows((2, 8, 1, 128), "bhnd", gen)
    want, _ = sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = q * 0
        late += q
        got, _ = sale.decode_attn(p, cache, late, prefix=prefix, prefix_len=64)
    side.synchronize()
    assert torch.equal(got, want)


def test_what_the_binding_refuses(sale):
    gen = torch.Generator().manual_seed(15)
    cache, prefix = make_cache(sale, [30, 20], 2, 16, "bf16", "bhnd", gen, 64)
    q = rows((2, 8, 1, 128), "bhnd", gen)
    p = sale.Params(2, 8, 2, 1)
    for args, kw in (((sale.Params(3, 8, 2, 1), cache, q), {}), ((sale.Params(2, 8, 4, 1), cache, q), {}), ((p, cache, q.float()), {}),
                     ((p, cache, q[:, :4]), {}), ((p, cache, q.cpu()), {}), ((p, cache, q), dict(prefix_len=10)),
                     ((p, cache, q), dict(prefix=prefix, prefix_len=65)), ((p, cache, q), dict(prefix=prefix.long(), prefix_len=64)),
                     ((p, cache, q), dict(prefix=prefix.cpu(), prefix_len=64)), ((p, cache, q), dict(out=q[:, :, :, :64])),
                     ((p, cache, q), dict(ws=torch.empty(10)))):
        with pytest.raises(ValueError):
            sale.decode_attn(*args, **kw)
    with pytest.raises(sale.SaleError):
        sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=64, ws=torch.empty(10, device="cuda"))
    k, v, t, n = cache.k, cache.v, cache.table, cache.lens
    for args in ((k.float(), v.float(), t, n), (k, v[:1], t, n), (k, v, t.long(), n), (k, v, t, n[:1]), (k, v, t[0], n), (k, v, t.cpu(), n),
                 (k.transpose(2, 3), v.transpose(2, 3), t, n), (bits(k).view(torch.float8_e4m3fn)[..., :128], bits(v).view(torch.float8_e4m3fn)[..., :128], t, n)):
        with pytest.raises(ValueError):
            sale.Cache(*args)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("batch,prefix_len,top_in,bad_in", [(1, 0, "own", "own"), (1, 700, "prefix", "own"), (1, 700, "own", "prefix"), (20, 1100, "own", "prefix"),
                                                            (20, 1100, "prefix", "own"), (1, 1100, "prefix", "prefix")])
def test_a_bad_value_that_is_seen_is_not_lost_in_the_join(sale, kind, batch, prefix_len, top_in, bad_in):
    """A NaN in V reaches every query that sees its key, also where another part of the keys has scores so much higher (by 500 and
    more) that its weight is zero in fp32; so does an infinity, as one or as zero times infinity."""
    gen = torch.Generator().manual_seed(17)
    cache, prefix = make_cache(sale, [3000] + [1500] * (batch - 1), 1, 16, kind, "bhnd", gen, prefix_len, spoil=False)
    cache.k.copy_(torch.zeros(cache.k.shape, dtype=torch.float32))
    if kind == "fp8":
        cache.k_scale.fill_(1.0)
    place = {"own": lambda pos: (int(cache.table[0, pos // 16]), 0, pos % 16), "prefix": lambda pos: (int(prefix[pos // 16]), 0, pos % 16)}
    value = torch.tensor(448.0).to(cache.k.dtype).cuda()
    bits(cache.k)[place[top_in](690) + (0,)] = bits(value)
    q = torch.zeros(batch, 4, 1, 128, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 16.0
    for value in ("nan",) + (("inf",) if kind == "bf16" else ()):
        bits(cache.v)[place[bad_in](5) + (slice(0, 128, 3),)] = bits(torch.tensor(float(value)).to(cache.v.dtype).cuda())
        o, lse = sale.decode_attn(sale.Params(batch, 4, 1, 1), cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
        assert not torch.isfinite(o[0, :, :, ::3]).any()
        keep = [c for c in range(128) if value == "nan" or c % 3]
        part = sale.Cache(cache.k, cache.v, cache.table[:1].contiguous(), cache.lens[:1].contiguous(), cache.k_scale, cache.v_scale)
        want = decode_oracle(part, q[:1], prefix, prefix_len)
        check(o[:1, ..., keep], lse[:1], [x[..., keep] if x.ndim == 4 else x for x in want])


def test_a_refused_cache_does_not_spoil_the_parameters(sale):
    """The workspace of a cache that the library refuses is 0 bytes; a good one under the same parameters has its own."""
    gen = torch.Generator().manual_seed(20)
    cache, _ = make_cache(sale, [900, 2000], 2, 16, "bf16", "bhnd", gen, spoil=False)
    p, q = sale.Params(2, 8, 2, 1), rows((2, 8, 1, 128), "bhnd", gen)
    apart = torch.zeros(cache.k.shape[0], 2, 16, 132, dtype=torch.bfloat16, device="cuda")[..., :128]      # (no multiple of 16 bytes)
    with pytest.raises(sale.SaleError):
        sale.decode_attn(p, sale.Cache(apart, apart, cache.table, cache.lens), q)
    o, lse = sale.decode_attn(p, cache, q, want_lse=True)
    check(o, lse, decode_oracle(cache, q, None, 0))
    short = sale.Cache(cache.k, cache.v, cache.table[:, :4].contiguous(), cache.lens)      # (left whole: no workspace)
    for c in (sale.Cache(apart, apart, short.table, short.lens), short):
        if c is short:
            o, lse = sale.decode_attn(p, c, q, want_lse=True)
            check(o, lse, decode_oracle(c, q, None, 0))
        else:
            with pytest.raises(sale.SaleError):
                sale.decode_attn(p, c, q)
        assert (0 in p._ws_bytes.values()) == (c is short)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("hq,lens,prefix_len,room", [(1, [40001], 20000, 1), (4, [32000], 16384, 1), (4, [66000], 0, 13000), (1, [66000], 16300, 13000)])
def test_more_parts_than_weights_at_a_time(sale, kind, hq, lens, prefix_len, room):
    """One KV head and one sequence: 250 .. 512 pieces of own keys (8-bit pages: 512 where the table has room for much), 79 or 128 parts of the prefix."""
    gen = torch.Generator().manual_seed(18)
    cache, prefix = make_cache(sale, lens, 1, 16, kind, "bhnd", gen, prefix_len, room=room, spoil=False)
    q = rows((1, hq, 1, 128), "bhnd", gen, 2.0)
    o, lse = sale.decode_attn(sale.Params(1, hq, 1, 1), cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    check(o, lse, decode_oracle(cache, q, prefix, prefix_len))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("page", [16, 64])
def test_a_query_that_is_not_finite_among_many_rows(sale, kind, page):
    """64 rows and more of a long prefix: the others' results keep their bits."""
    gen = torch.Generator().manual_seed(19)
    batch, prefix_len = 40, 5000
    cache, prefix = make_cache(sale, [5] * batch, 1, page, kind, "bhnd", gen, prefix_len)
    p, q = sale.Params(batch, 4, 1, 1), rows((batch, 4, 1, 128), "bhnd", gen, 2.0)
    clean, clean_lse = sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    hit = torch.zeros(batch, 4, 1, dtype=torch.bool, device="cuda")
    for s, h, value in ((0, 1, "nan"), (17, 2, "inf"), (18, 0, "-inf"), (39, 3, "nan")):
        q[s, h, 0, 5], hit[s, h, 0] = float(value), True
    o, lse = sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    assert torch.isnan(o[hit]).all()
    assert torch.equal(o[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("batch,n,prefix_len", [(3, 1, 0), (3, 6, 40), (33, 2, 2100)])
def test_keys_and_values_of_different_layouts(sale, kind, batch, n, prefix_len):
    gen = torch.Generator().manual_seed(21)
    lens = [1000, 0, 77] * (batch // 3)
    cache, prefix = make_cache(sale, lens, 2, 32, kind, "padded", gen, prefix_len)
    v = bits(cache.v).transpose(1, 2).contiguous().transpose(1, 2).view(cache.v.dtype)
    q = rows((batch, 8, n, 128), "bnhd", gen, 2.0)
    p = sale.Params(batch, 8, 2, n)
    for c in (sale.Cache(cache.k, v, cache.table, cache.lens, cache.k_scale, cache.v_scale),
              sale.Cache(bits(cache.k).contiguous().view(cache.k.dtype), v, cache.table, cache.lens, cache.k_scale, cache.v_scale)):
        o, lse = sale.decode_attn(p, c, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
        _some(sale, c, q, o, lse, prefix, prefix_len, [0, 1, batch - 1])
        assert torch.equal(o, sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=prefix_len)[0])


@pytest.mark.parametrize("n", [1, 5])
@pytest.mark.parametrize("prefix_len", [0, 50])
def test_a_batch_that_holds_nothing(sale, n, prefix_len):
    """Under a table with room for much: every sequence empty; then one token in the last one."""
    gen = torch.Generator().manual_seed(22)
    cache, prefix = make_cache(sale, [0] * 9, 2, 16, "bf16", "bhnd", gen, prefix_len, room=300)
    p, q = sale.Params(9, 8, 2, n), rows((9, 8, n, 128), "bhnd", gen)
    for last in (0, 1):
        if last:
            cache.table[8, 0] = 0
            cache.k[0], cache.v[0] = 1.0, 2.0
            cache.lens[8] = 1
        o, lse = sale.decode_attn(p, cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
        check(o, lse, decode_oracle(cache, q, prefix, prefix_len))
        if prefix_len == 0:
            assert bool((o[:8] == 0).all() and (lse[:8] == -float("inf")).all())


def _bound_by_largest(o, slack, most):
    """As the oracle's, with the largest |v| in the place of the average."""
    return 2.0 ** -8 * (2 * np.abs(o) + most) + 2 * slack[..., None] * most


@pytest.mark.parametrize("batch,n,prefix_len,at", [(1, 1, 0, "own"), (3, 1, 1100, "prefix"), (3, 1, 1100, "own"), (20, 1, 1100, "prefix"), (20, 1, 1100, "own"), (3, 6, 300, "prefix")])
@pytest.mark.parametrize("value", ["nan", "inf", "-inf"])
def test_a_key_that_is_seen_and_not_finite(sale, batch, n, prefix_len, at, value):
    """A score of NaN or infinity makes O and lse NaN; one of minus infinity has no weight."""
    gen = torch.Generator().manual_seed(23)
    cache, prefix = make_cache(sale, [1500] + [40] * (batch - 1), 1, 16, "bf16", "bhnd", gen, prefix_len, spoil=False)
    pos = min(200, prefix_len - 1) if at == "prefix" else 700
    cache.k[int(prefix[pos // 16]) if at == "prefix" else int(cache.table[0, pos // 16]), 0, pos % 16, 5] = float(value)
    q = rows((batch, 4, n, 128), "bhnd", gen, 2.0)
    q[:, :2, :, 5], q[:, 2:, :, 5] = 1.5, -1.5
    o, lse = sale.decode_attn(sale.Params(batch, 4, 1, n), cache, q, prefix=prefix, prefix_len=prefix_len, want_lse=True)
    part = sale.Cache(cache.k, cache.v, cache.table[:1].contiguous(), cache.lens[:1].contiguous())
    want = decode_oracle(part, q[:1], prefix, prefix_len)
    lost = np.isnan(want[0][0, :, 0, 0])
    assert lost.tolist() == {"nan": [True] * 4, "inf": [True, True, False, False], "-inf": [False, False, True, True]}[value]
    assert torch.isnan(o[0, lost]).all() and torch.isnan(lse[0, lost]).all()
    sound = ~lost
    if sound.any():
        # (the bound without the key itself, whose size is infinite)
        cache.k[int(prefix[pos // 16]) if at == "prefix" else int(cache.table[0, pos // 16]), 0, pos % 16, 5] = 0.0
        slack = decode_oracle(part, q[:1], prefix, prefix_len)[3]
        tol = _bound_by_largest(want[0], slack, f64(cache.v).__abs__().max())
        got = f64(o[:1])[:, sound]
        assert (np.abs(got - want[0][:, sound]) <= tol[:, sound]).all()
        assert (np.abs(f64(lse[:1])[:, sound] - want[1][:, sound]) <= slack[:, sound] + np.abs(want[1][:, sound]) * 2.0 ** -22 + 2.0 ** -20).all()
