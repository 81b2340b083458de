"""Caches and inputs for the tests of the serving calls."""
import numpy as np
import torch

from oracle import serving_oracle as so


def f64(x):
    return x.detach().cpu().to(torch.float32 if x.element_size() == 1 else x.dtype).double().numpy()


def rows(shape, layout, gen, scale=1.0):
    """bf16 [B, H, N, d] on the GPU: contiguous, as a view of [B, N, H, d], or inside a larger tensor with NaN around it."""
    b, h, n, d = shape
    x = (torch.randn(shape, generator=gen) * scale).bfloat16().cuda()
    if layout == "bnhd":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "padded":
        big = torch.full((b + 1, h + 2, n + 3, d + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
        big[:b, :h, 1:n + 1, 8:d + 8] = x
        return big[:b, :h, 1:n + 1, 8:d + 8]
    return x


def pool(n_pages, hkv, page, kind, layout, gen, scale):
    """Pages of bf16 or E4M3, contiguous or as a view of [page][token][head][d], or with gaps."""
    x = torch.randn(n_pages, hkv, page, 128, generator=gen).cuda()
    x = x.bfloat16() if kind == "bf16" else (x / scale.cuda()[:, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    bits = x.view(torch.int16 if kind == "bf16" else torch.uint8)
    if layout == "bnhd":
        bits = bits.transpose(1, 2).contiguous().transpose(1, 2)
    elif layout == "padded":
        big = torch.full((n_pages, hkv + 1, page + 2, 160), -1 if kind == "bf16" else 255, dtype=bits.dtype, device="cuda")      # (NaN)
        big[:, :hkv, :page, :128] = bits
        bits = big[:, :hkv, :page, :128]
    return bits.view(x.dtype)


def bits(x):
    return x.view(torch.uint8 if x.element_size() == 1 else torch.int16)


def make_cache(sale, lens, hkv, page, kind, layout, gen, prefix_len=0, room=1, spoil=True):
    """A cache whose sequences hold `lens` tokens in scattered pages, and the pages of a prefix.  spoil: what is no key is NaN."""
    need = [-(-max(n, 0) // page) for n in lens]
    n_prefix = -(-prefix_len // page)
    n_pages = sum(need) + n_prefix + 3
    order = torch.randperm(n_pages, generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(need) + room), -1, dtype=torch.int32)
    used = 0
    for s, n in enumerate(need):
        table[s, :n] = order[used:used + n]
        used += n
    prefix = order[used:used + n_prefix].contiguous()
    scale = 0.01 + 0.02 * torch.rand(2, hkv, generator=gen)
    k, v = (pool(n_pages, hkv, page, kind, layout, gen, scale[i]) for i in range(2))
    if spoil:
        holds = torch.zeros(n_pages, page, dtype=torch.bool)
        for s, n in enumerate(lens):
            for i in range(max(n, 0)):
                holds[int(table[s, i // page]), i % page] = True
        for i in range(prefix_len):
            holds[int(prefix[i // page]), i % page] = True
        at, slot = (~holds).nonzero(as_tuple=True)
        for x in (k, v):
            bits(x)[at.cuda(), :, slot.cuda()] = -1 if kind == "bf16" else 255
    scales = dict(k_scale=scale[0].cuda(), v_scale=scale[1].cuda()) if kind == "fp8" else {}
    cache = sale.Cache(k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), **scales)
    return cache, prefix.cuda()


def decode_oracle(cache, q, prefix, prefix_len):
    k, v = f64(cache.k), f64(cache.v)
    if cache.k_scale is not None:
        k, v = k * f64(cache.k_scale)[:, None, None], v * f64(cache.v_scale)[:, None, None]
    pages = np.zeros(0, dtype=np.int64) if prefix is None else prefix.cpu().numpy()
    return so.decode(f64(q), k, v, cache.table.cpu().numpy(), cache.lens.cpu().numpy(), pages, prefix_len)


def check(o, lse, want, rounded_sums=False):
    """Against the oracle's O, lse, bound of O and slack; not finite where the oracle is not."""
    ref, ref_lse, tol, slack = want
    got = f64(o)
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), "NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
    off = np.abs(got[fine] - ref[fine]) - tol[fine]
    assert off.size == 0 or off.max() <= 0, f"{(off > 0).sum()} of {off.size} values off, worst by {off.max():.3g} beyond {tol[fine][off.argmax()]:.3g}"
    if lse is None:
        return
    got = f64(lse)
    assert np.array_equal(got == -np.inf, ref_lse == -np.inf)
    fine = np.isfinite(ref_lse)
    room = slack[fine] + np.abs(ref_lse[fine]) * 2.0 ** -22 + 2.0 ** -20 + (so.EPS if rounded_sums else 0)
    off = np.abs(got[fine] - ref_lse[fine]) - room
    assert off.size == 0 or off.max() <= 0, f"lse off by {off.max():.3g} beyond its bound"
