"""cache_append and cache_copy: every byte of the pages against what the definition says, written or left alone."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from serving_utils import bits, f64, make_cache, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sale():
    from paper_2505_24179_amd import sale as mod
    return mod


def _expected(cache, x, side, new):
    """The pool after the append, as bits: x [tokens in packed order, Hkv, d] on the CPU."""
    pool = bits(getattr(cache, side)).cpu().clone()
    page, fp8 = cache.k.shape[2], cache.k.dtype == torch.float8_e4m3fn
    table, starts = cache.table.cpu(), np.concatenate([[0], np.cumsum(new)])
    if fp8:
        scale = getattr(cache, side + "_scale").cpu()
        y = (x.float() / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        assert np.array_equal(so.e4m3(x.float().numpy() / scale.numpy()[:, None]), y.double().numpy(), equal_nan=True)
        x = y
    for s, i, pos in so.positions(cache.lens.tolist(), new):
        if pos // page < table.shape[1] and 0 <= int(table[s, pos // page]) < pool.shape[0]:
            pool[int(table[s, pos // page]), :, pos % page] = bits(x)[starts[s] + i]
    return pool


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd", "padded"])
@pytest.mark.parametrize("hkv,page,batch,n", [(1, 16, 1, 1), (8, 16, 5, 1), (2, 32, 3, 7), (3, 64, 2, 100), (70, 16, 2, 3), (2, 256, 1, 333)])
def test_append_to_a_batch(sale, kind, layout, hkv, page, batch, n):
    gen = torch.Generator().manual_seed(hkv * 100 + page + n)
    held = [int(x) for x in torch.randint(0, 90, (batch,), generator=gen)]
    held[0] = 0
    cache, _ = make_cache(sale, [h + n for h in held], hkv, page, kind, layout, gen)
    k, v = rows((batch, hkv, n, 128), layout, gen, 3.0), rows((batch, hkv, n, 128), layout, gen, 3.0)
    want = [_expected(cache, x.transpose(1, 2).flatten(0, 1).cpu(), side, [n] * batch) for x, side in ((k, "k"), (v, "v"))]
    sale.cache_append(sale.Params(batch, hkv * 2, hkv, n), cache, k, v)
    for x, side in zip(want, ("k", "v")):
        assert torch.equal(bits(getattr(cache, side)).cpu(), x), side


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_append_packed_sequences(sale, kind, layout):
    gen = torch.Generator().manual_seed(3)
    new = [5, 0, 1, 64, 17, 0, 130] + [1, 2, 0] * 100      # (more sequences than travel with one launch)
    held = [int(x) for x in torch.randint(0, 40, (len(new),), generator=gen)]
    cache, _ = make_cache(sale, [h + n for h, n in zip(held, new)], 2, 16, kind, "bhnd", gen)
    total = sum(new)
    k, v = rows((1, 2, total, 128), layout, gen, 3.0), rows((1, 2, total, 128), layout, gen, 3.0)
    want = [_expected(cache, x.transpose(1, 2).flatten(0, 1).cpu(), side, new) for x, side in ((k, "k"), (v, "v"))]
    p = sale.Params(1, 4, 2, total, cu_seqlens=tuple(int(x) for x in np.concatenate([[0], np.cumsum(new)])))
    sale.cache_append(p, cache, k, v)
    for x, side in zip(want, ("k", "v")):
        assert torch.equal(bits(getattr(cache, side)).cpu(), x), side


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_tokens_without_a_place_are_dropped(sale, kind):
    gen = torch.Generator().manual_seed(4)
    cache, _ = make_cache(sale, [40, 40, 40, 40, 40], 2, 16, kind, "bhnd", gen, room=0)
    cache.lens.copy_(torch.tensor([3, -9, 2 ** 31 - 1, 52, 0], dtype=torch.int32))      # partly negative, negative, far beyond, partly beyond
    cache.table[0, 0], cache.table[3, 2] = cache.k.shape[0], -2 ** 31
    k, v = rows((5, 2, 8, 128), "bhnd", gen), rows((5, 2, 8, 128), "bhnd", gen)
    want = [_expected(cache, x.transpose(1, 2).flatten(0, 1).cpu(), side, [8] * 5) for x, side in ((k, "k"), (v, "v"))]
    sale.cache_append(sale.Params(5, 4, 2, 8), cache, k, v)
    for x, side in zip(want, ("k", "v")):
        assert torch.equal(bits(getattr(cache, side)).cpu(), x), side


def test_values_that_8_bits_cannot_hold(sale):
    gen = torch.Generator().manual_seed(5)
    cache, _ = make_cache(sale, [4], 1, 16, "fp8", "bhnd", gen)
    x = torch.zeros(1, 1, 4, 128, dtype=torch.bfloat16)
    x[0, 0, 0, :8] = torch.tensor([float("inf"), -float("inf"), float("nan"), 1e30, -1e30, 0.0, -0.0, 1e-30])
    x[0, 0, 1] = torch.linspace(-20, 20, 128)
    x[0, 0, 2] = torch.linspace(-0.01, 0.01, 128)      # subnormal codes and their ties
    x = x.cuda()
    sale.cache_append(sale.Params(1, 1, 1, 4), cache, x, x)
    got = f64(cache.k)[int(cache.table[0, 0]), 0, :4]
    want = so.e4m3(x.cpu().float().numpy()[0, 0] / cache.k_scale.cpu().numpy())
    assert np.array_equal(got, want, equal_nan=True)
    assert got[0, 0] == 448 and got[0, 1] == -448 and np.isnan(got[0, 2]) and got[0, 3] == 448


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd", "padded"])
@pytest.mark.parametrize("hkv,page", [(1, 16), (3, 16), (8, 64), (2, 256)])
def test_copy(sale, kind, layout, hkv, page):
    gen = torch.Generator().manual_seed(hkv + page)
    cache, _ = make_cache(sale, [page * 30], hkv, page, kind, layout, gen, spoil=False)
    n_pages = cache.k.shape[0]
    order = torch.randperm(n_pages, generator=gen).tolist()
    src, dst = [order[0], order[1], order[0], order[2]], order[3:7]
    before = [bits(x).clone() for x in (cache.k, cache.v)]
    sale.cache_copy(sale.Params(1, hkv, hkv, 1), cache, src, dst)
    for x, old in zip((cache.k, cache.v), before):
        want = old.clone()
        want[dst] = old[src]
        assert torch.equal(bits(x), want)
    if layout == "padded":      # the gaps between the pages' rows are left alone
        for x in (cache.k, cache.v):
            base = bits(x)
            whole = torch.as_strided(base, (n_pages, hkv + 1, page + 2, 160), base.stride(), 0)
            fill = -1 if kind == "bf16" else 255
            assert bool((whole[:, hkv] == fill).all() and (whole[:, :, page:] == fill).all() and (whole[..., 128:] == fill).all())


def test_copy_of_many_pages_and_none(sale):
    gen = torch.Generator().manual_seed(6)
    cache, _ = make_cache(sale, [16 * 2000], 1, 16, "bf16", "bhnd", gen, spoil=False)
    order = torch.randperm(2000, generator=gen).to(torch.int32)
    old = bits(cache.k).clone()
    p = sale.Params(1, 1, 1, 1)
    sale.cache_copy(p, cache, [], [])
    assert torch.equal(bits(cache.k), old)
    src, dst = order[:1000].contiguous(), order[1000:].contiguous()      # (more than travel with one launch)
    sale.cache_copy(p, cache, src, dst)
    want = old.clone()
    want[dst.long()] = old[src.long()]
    assert torch.equal(bits(cache.k), want)


def test_what_the_binding_refuses(sale):
    gen = torch.Generator().manual_seed(7)
    cache, _ = make_cache(sale, [30, 20], 2, 16, "bf16", "bhnd", gen)
    p, k = sale.Params(2, 4, 2, 3), rows((2, 2, 3, 128), "bhnd", gen)
    for args in ((sale.Params(1, 4, 2, 3), cache, k[:1], k[:1]), (p, cache, k[:, :, :2], k), (p, cache, k, k.half()), (p, cache, k.cpu(), k)):
        with pytest.raises(ValueError):
            sale.cache_append(*args)
    for src, dst in (([0], [1, 2]), (torch.zeros(1, dtype=torch.int64), torch.ones(1, dtype=torch.int64)),
                     (torch.zeros(1, dtype=torch.int32).cuda(), torch.ones(1, dtype=torch.int32).cuda())):
        with pytest.raises(ValueError):
            sale.cache_copy(p, cache, src, dst)
    for src, dst in (([0], [0]), ([0, 1], [2, 2]), ([0], [99]), ([-1], [1])):
        with pytest.raises(sale.SaleError):
            sale.cache_copy(p, cache, src, dst)


@pytest.mark.parametrize("page", [16, 64])
def test_zero_keeps_its_sign_in_8_bits(sale, page):
    """The codes of zeros and of what rounds to zero, as bits: those of IEEE division and rounding."""
    gen = torch.Generator().manual_seed(8)
    cache, _ = make_cache(sale, [4], 2, page, "fp8", "bhnd", gen)
    cache.k_scale.copy_(torch.tensor([0.011, 3.0]))
    cache.v_scale.copy_(torch.tensor([1e-25, 1e25]))      # (beyond the range of the quick quotient)
    x = torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16)
    x[..., 0, 1::2] = -0.0
    x[..., 1, :] = torch.tensor([-1e-40, 1e-40] * 64)
    x[..., 2, :] = torch.linspace(-1e-4, 1e-4, 128)
    x[..., 3, :] = torch.tensor([-0.0, -1.0] * 64)
    want = [_expected(cache, x[0].transpose(0, 1), side, [4]) for side in ("k", "v")]
    sale.cache_append(sale.Params(1, 4, 2, 4), cache, x.cuda(), x.cuda())
    for side, w in zip(("k", "v"), want):
        assert torch.equal(bits(getattr(cache, side)).cpu(), w), side
    assert int((want[0] == 128).sum()) > 64
