"""prompt_attn: prompts of any lengths against the oracle, and against dense_attn where that takes them too."""
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


def _want(q, k, v, offsets, b=0):
    return [x[None] for x in so.prompt(f64(q)[b], f64(k)[b], f64(v)[b], offsets)]


@pytest.mark.parametrize("hq,hkv,layout", [(1, 1, "bhnd"), (6, 2, "bnhd"), (4, 1, "padded"), (3, 3, "bhnd")])
@pytest.mark.parametrize("n", [1, 2, 31, 33, 63, 64, 65, 127, 129, 200])
def test_one_length(sale, hq, hkv, layout, n):
    gen = torch.Generator().manual_seed(n * 10 + hq)
    q, k, v = (rows((2, h, n, 128), layout, gen, s) for h, s in ((hq, 2.0), (hkv, 1.0), (hkv, 1.0)))
    o, lse = sale.prompt_attn(sale.Params(2, hq, hkv, n), q, k, v, want_lse=True)
    for b in range(2):
        check(o[b:b + 1], lse[b:b + 1], _want(q, k, v, [0, n], b), rounded_sums=True)


@pytest.mark.parametrize("layout", ["bhnd", "bnhd", "padded"])
def test_packed_lengths(sale, layout):
    gen = torch.Generator().manual_seed(5)
    new = [3, 0, 64, 1, 130, 65, 0, 0, 17, 63, 1]
    offsets = tuple(int(x) for x in np.concatenate([[0], np.cumsum(new)]))
    q, k, v = (rows((1, h, offsets[-1], 128), layout, gen) for h in (4, 2, 2))
    p = sale.Params(1, 4, 2, offsets[-1], cu_seqlens=offsets)
    o, lse = sale.prompt_attn(p, q, k, v, want_lse=True)
    check(o, lse, _want(q, k, v, offsets), rounded_sums=True)


def test_many_sequences(sale):
    """More than travel with one launch, empty ones at both ends of a chunk."""
    gen = torch.Generator().manual_seed(6)
    new = [0, 0] + [int(x) for x in torch.randint(0, 9, (600,), generator=gen)] + [70, 0, 0]
    new[250:260] = [0] * 10
    offsets = tuple(int(x) for x in np.concatenate([[0], np.cumsum(new)]))
    q, k, v = (rows((1, h, offsets[-1], 128), "bhnd", gen) for h in (2, 1, 1))
    o, lse = sale.prompt_attn(sale.Params(1, 2, 1, offsets[-1], cu_seqlens=offsets), q, k, v, want_lse=True)
    check(o, lse, _want(q, k, v, offsets), rounded_sums=True)


@pytest.mark.parametrize("lengths,hq,hkv", [((2048,), 4, 1), ((64, 1024, 192), 8, 2), ((4096,), 32, 8), ((1024,) * 40, 1, 1)])
def test_the_same_bits_as_the_dense_call(sale, lengths, hq, hkv):
    gen = torch.Generator().manual_seed(7)
    n = sum(lengths)
    offsets = tuple(int(x) for x in np.concatenate([[0], np.cumsum(lengths)]))
    q, k, v = (rows((1, h, n, 128), "bhnd", gen) for h in (hq, hkv, hkv))
    p = sale.Params(1, hq, hkv, n, cu_seqlens=offsets if len(lengths) > 1 else ())
    o, lse = sale.prompt_attn(p, q, k, v, want_lse=True)
    want, want_lse = sale.dense_attn(p, q, k, v, want_lse=True)
    assert torch.equal(o, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("n,hq,hkv", [(1500, 4, 1), (5001, 16, 8), (9999, 6, 2)])
def test_a_sequence_does_not_depend_on_its_place(sale, n, hq, hkv):
    """Alone, and behind and in front of others: the same up to the rounding of two forms of the kernel; rows in between checked."""
    gen = torch.Generator().manual_seed(8)
    q, k, v = (rows((1, h, n + 100, 128), "bhnd", gen) for h in (hq, hkv, hkv))
    o, _ = sale.prompt_attn(sale.Params(1, hq, hkv, n + 100, cu_seqlens=(0, 37, 37 + n, n + 100)), q, k, v)
    mine = [x[:, :, 37:37 + n] for x in (q, k, v)]
    alone, _ = sale.prompt_attn(sale.Params(1, hq, hkv, n), *mine)
    assert torch.equal(alone, o[:, :, 37:37 + n])
    some = [0, 63, 64, n // 2, n - 2, n - 1]
    seen = np.arange(n)[None] <= np.array(some)[:, None]
    for h in (0, hq - 1):
        want = so.attend(f64(mine[0])[0, h, some], f64(mine[1])[0, h // (hq // hkv)], f64(mine[2])[0, h // (hq // hkv)], seen)
        check(alone[0, h, some], None, want)


def test_rows_sorted_by_length(sale):
    """More sequences than travel with one launch, few enough rows that they are sorted: as in calls of a few of them."""
    gen = torch.Generator().manual_seed(14)
    new = [int(x) for x in torch.randint(193, 257, (300,), generator=gen)]
    offsets = [int(x) for x in np.concatenate([[0], np.cumsum(new)])]
    q, k, v = (rows((1, 1, offsets[-1], 128), "bhnd", gen) for _ in range(3))
    o, lse = sale.prompt_attn(sale.Params(1, 1, 1, offsets[-1], cu_seqlens=tuple(offsets)), q, k, v, want_lse=True)
    for a in range(0, 300, 60):
        t0, t1 = offsets[a], offsets[a + 60]
        p = sale.Params(1, 1, 1, t1 - t0, cu_seqlens=tuple(x - t0 for x in offsets[a:a + 61]))
        part, part_lse = sale.prompt_attn(p, q[:, :, t0:t1], k[:, :, t0:t1], v[:, :, t0:t1], want_lse=True)
        assert torch.equal(o[:, :, t0:t1], part) and torch.equal(lse[:, :, t0:t1], part_lse)


@pytest.mark.parametrize("hq,hkv,n", [(2, 1, 75), (4, 4, 200)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_later_token_that_is_not_finite(sale, hq, hkv, n, value):
    """In K and V: queries before it do not see it.  (In the block of the query itself, where it is one of the masked keys.)"""
    gen = torch.Generator().manual_seed(9)
    q, k, v = (rows((1, h, n, 128), "bhnd", gen) for h in (hq, hkv, hkv))
    clean, clean_lse = sale.prompt_attn(sale.Params(1, hq, hkv, n), q, k, v, want_lse=True)
    for at in (1, 40, 66, n - 1):
        k2, v2 = k.clone(), v.clone()
        v2[:, :, at, ::5] = value
        o, lse = sale.prompt_attn(sale.Params(1, hq, hkv, n), q, k2, v2, want_lse=True)
        check(o[:, :, :at], None, [x[:, :, :at] for x in _want(q, k, v, [0, n])])
        assert torch.equal(lse, clean_lse)
        assert not torch.isfinite(o[:, :, at:, ::5]).any()
        keep = [c for c in range(128) if c % 5]
        check(o[..., keep], None, [x[..., keep] if x.ndim == 4 else x for x in _want(q, k, v, [0, n])])
        k2[:, :, at] = value
        o, lse = sale.prompt_attn(sale.Params(1, hq, hkv, n), q, k2, v2, want_lse=True)
        check(o[:, :, :at], lse[:, :, :at], [x[:, :, :at] for x in _want(q, k, v, [0, n])], rounded_sums=True)


def test_nothing_beyond_the_outputs_is_written(sale):
    gen = torch.Generator().manual_seed(10)
    offsets = (0, 70, 70, 101)
    q, k, v = (rows((1, h, 101, 128), "padded", gen) for h in (4, 2, 2))
    p = sale.Params(1, 4, 2, 101, cu_seqlens=offsets)
    plain, _ = sale.prompt_attn(p, q, k, v)
    big = torch.full((1, 6, 140, 160), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[:, 1:5, 20:121, 16:144]
    need = sale.workspace_bytes(p, sale.WS_PROMPT_ATTN)
    ws = torch.full((need + 4096,), 173, dtype=torch.uint8, device="cuda")
    sale.prompt_attn(p, q, k, v, out=out, ws=ws[:need])
    assert torch.equal(out, plain) and bool((ws[need:] == 173).all())
    out.fill_(7.0)
    assert bool((big == 7.0).all())


def test_captured(sale):
    gen = torch.Generator().manual_seed(11)
    offsets = (0, 333, 334, 900)
    q, k, v = (rows((1, h, 900, 128), "bhnd", gen) for h in (8, 2, 2))
    p = sale.Params(1, 8, 2, 900, cu_seqlens=offsets)
    o, ws = torch.empty_like(q), torch.empty(sale.workspace_bytes(p, sale.WS_PROMPT_ATTN), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sale.prompt_attn(p, q, k, v, out=o, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sale.prompt_attn(p, q, k, v, out=o, ws=ws)
    for _ in range(3):
        for x, h in ((q, 8), (k, 2), (v, 2)):
            x.copy_(rows((1, h, 900, 128), "bhnd", gen))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, sale.prompt_attn(p, q, k, v)[0])


def test_what_the_binding_refuses(sale):
    gen = torch.Generator().manual_seed(12)
    q, k = rows((1, 4, 50, 128), "bhnd", gen), rows((1, 2, 50, 128), "bhnd", gen)
    p = sale.Params(1, 4, 2, 50)
    for args in ((p, q, k, k[:, :, :49]), (p, q.half(), k, k), (p, q.cpu(), k, k), (p, q, k, None), (sale.Params(1, 4, 2, 51), q, k, k)):
        with pytest.raises(ValueError):
            sale.prompt_attn(*args)
    with pytest.raises(sale.SaleError):
        sale.prompt_attn(sale.Params(1, 4, 2, 50, flags=sale.FLAG_ATTN_INT8_QK), q, k, k)
    with pytest.raises(sale.SaleError):
        sale.prompt_attn(p, q, k, k, ws=torch.empty(100, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("offsets,hq,hkv", [((0, 2751), 32, 8), ((0, 1309, 1310, 3001), 32, 8)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_later_token_that_is_not_finite_in_a_large_call(sale, offsets, hq, hkv, value):
    """As above, with more rows than two waves per row are taken for; in a sequence's last block, which is partly filled, too."""
    gen = torch.Generator().manual_seed(15)
    n, t0 = offsets[-1], offsets[-2]
    q, k, v = (rows((1, h, n, 128), "bhnd", gen) for h in (hq, hkv, hkv))
    p = sale.Params(1, hq, hkv, n, cu_seqlens=offsets if len(offsets) > 2 else ())
    clean, clean_lse = sale.prompt_attn(p, q, k, v, want_lse=True)
    for at in (t0 + 70, n - 9, n - 1):
        k2, v2 = k.clone(), v.clone()
        v2[:, :, at, ::5] = value
        o, lse = sale.prompt_attn(p, q, k, v2, want_lse=True)
        block = t0 + (at - t0) // 64 * 64
        assert torch.equal(lse, clean_lse) and torch.equal(o[:, :, :block], clean[:, :, :block])
        assert not torch.isfinite(o[:, :, at:, ::5]).any() and torch.isfinite(o[:, :, :at]).all()
        some = sorted({block, at - 1, at, n - 1})
        seen = np.arange(n - t0)[None] <= np.array(some)[:, None] - t0
        keep = [c for c in range(128) if c % 5]
        for h in (0, hq - 1):
            want = so.attend(f64(q)[0, h, some], f64(k)[0, h * hkv // hq, t0:], f64(v)[0, h * hkv // hq, t0:], seen)
            check(o[0, h, some][:, keep], None, [x[:, keep] if x.ndim == 2 else x for x in want])
            before = [i for i, t in enumerate(some) if t < at]
            check(o[0, h, some][before], None, [x[before] for x in want])
        k2[:, :, at] = value
        o, lse = sale.prompt_attn(p, q, k2, v2, want_lse=True)
        assert torch.equal(o[:, :, :block], clean[:, :, :block]) and torch.equal(lse[:, :, :at], clean_lse[:, :, :at])
        assert torch.isfinite(o[:, :, :at]).all()


@pytest.mark.parametrize("n,hq,hkv", [(900, 2, 1), (2751, 32, 8)])
def test_an_earlier_value_that_is_not_finite_is_not_lost(sale, n, hq, hkv):
    """Behind it, scores so much higher that its probabilities are zero in fp32; and beside sequences that it is not part of."""
    gen = torch.Generator().manual_seed(16)
    q, k, v = (torch.zeros(1, h, n, 128, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    q[..., 0] = 16.0
    k[:, :, 50, 0] = 20.0
    k[:, :, 600, 0] = 400.0
    v.copy_(rows((1, hkv, n, 128), "bhnd", gen))
    v[:, :, 3, ::7] = float("nan")
    offsets = (0, 1, n - 130, n)
    for offs in ((), offsets):
        p = sale.Params(1, hq, hkv, n, cu_seqlens=offs)
        o, _ = sale.prompt_attn(p, q, k, v)
        end = n if not offs else n - 130
        assert torch.isnan(o[:, :, 3:end, ::7]).all() and torch.isfinite(o[:, :, :3]).all() and torch.isfinite(o[:, :, end:]).all()
        keep = [c for c in range(128) if c % 7]
        assert torch.isfinite(o[..., keep]).all()
