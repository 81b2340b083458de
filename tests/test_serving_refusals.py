"""What the serving calls refuse, before anything is launched: through the C ABI with pointers that are never followed, and in
the binding's own checks."""
import ctypes

import pytest
import torch

F = ctypes.c_void_p(0x1000)


@pytest.fixture(scope="module")
def sale():
    from paper_2505_24179_amd import sale as mod
    return mod


def _cache(sale, **kw):
    c = sale._Cache(k=0x1000, v=0x1000, n_pages=10, page_tokens=16, dtype=0, table_width=4, table=0x1000, lens=0x1000)
    for name, x in kw.items():
        if name.endswith("stride"):
            getattr(c, name)[:] = x
        else:
            setattr(c, name, x)
    return c


def _params(sale, batch=2, hq=8, hkv=2, n=1, **kw):
    p = sale.Params(batch, hq, hkv, n, **{k: v for k, v in kw.items() if not k.endswith("_stride")})
    c = p.c()
    for name in kw:
        if name.endswith("_stride"):
            getattr(c, name)[:] = kw[name]
    return c


BAD_PARAMS = [(dict(batch=0), -2), (dict(n=0), -2), (dict(n=-1), -2), (dict(hq=7), -2), (dict(hkv=0), -2), (dict(head_dim=64), -3),
              (dict(flags=8), -3), (dict(flags=32), -3), (dict(cu_seqlens=(0, 1)), -2), (dict(batch=1, n=3, cu_seqlens=(0, 2, 1, 3)), -2),
              (dict(batch=1, n=3, cu_seqlens=(0, 2)), -2), (dict(batch=1, n=3, cu_seqlens=(1, 3)), -2)]


@pytest.mark.parametrize("kw,status", BAD_PARAMS)
def test_parameters(sale, kw, status):
    lib, p, c = sale.raw(), _params(sale, **kw), _cache(sale)
    b = ctypes.byref
    assert lib.sale_prompt_attn(b(p), F, F, F, F, None, F, 1 << 40, None) == status
    assert lib.sale_workspace_bytes(b(p), sale.WS_PROMPT_ATTN) == 0
    assert lib.sale_cache_append(b(p), b(c), F, F, None) == status
    assert lib.sale_decode_attn(b(p), b(c), F, None, 0, F, None, F, 1 << 40, None) == status
    assert lib.sale_decode_workspace_bytes(b(p), b(c), 0) == 0


@pytest.mark.parametrize("stride", [(128, 64, 4), (0, 128, 128), (1024, 0, 128), (1024, 128, 64), (1024, 129, 128), (1024, -128, 128)])
def test_strides(sale, stride):
    lib, c, b = sale.raw(), _cache(sale), ctypes.byref
    p = _params(sale, q_stride=stride)
    assert lib.sale_prompt_attn(b(p), F, F, F, F, None, F, 1 << 40, None) == -2
    assert lib.sale_decode_attn(b(p), b(c), F, None, 0, F, None, F, 1 << 40, None) == -2
    p = _params(sale, k_stride=stride)
    assert lib.sale_cache_append(b(p), b(c), F, F, None) == -2


BAD_CACHE = [(dict(k=None), -1), (dict(v=None), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(n_pages=0), -2),
             (dict(table_width=0), -2), (dict(page_tokens=0), -2), (dict(page_tokens=8), -3), (dict(page_tokens=48), -3),
             (dict(page_tokens=512), -3), (dict(dtype=2), -3), (dict(dtype=1), -1), (dict(dtype=1, k_scale=0x1000), -1),
             (dict(k=0x1008), -2), (dict(v=0x1002), -2), (dict(k_stride=(4096, 2048, 64)), -2), (dict(v_stride=(4096, 2048, 132)), -2),
             (dict(k_stride=(4096, 0, 128)), -2), (dict(v_stride=(0, 2048, 128)), -2), (dict(k_stride=(4096, 2048, (1 << 22) + 8)), -3), (dict(v_stride=(1 << 31, 2048, 128)), -3),
             (dict(k_stride=(-4096, 2048, 128)), -2), (dict(dtype=1, k_scale=0x1000, v_scale=0x1000, k_stride=(4096, 2048, 136)), -2),
             (dict(table_width=1 << 28), -3)]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_caches(sale, kw, status):
    lib, p, c, b = sale.raw(), _params(sale), _cache(sale, **kw), ctypes.byref
    assert lib.sale_cache_append(b(p), b(c), F, F, None) == status
    assert lib.sale_decode_attn(b(p), b(c), F, None, 0, F, None, F, 1 << 40, None) == status
    assert lib.sale_decode_workspace_bytes(b(p), b(c), 0) == 0


def test_null_and_misaligned_tensors(sale):
    lib, p, c, b = sale.raw(), _params(sale), _cache(sale), ctypes.byref
    odd = ctypes.c_void_p(0x1004)
    for at in range(4):
        args = [F, F, F, F]
        args[at] = None
        assert lib.sale_prompt_attn(b(p), *args, None, F, 1 << 40, None) == -1
        args[at] = odd
        assert lib.sale_prompt_attn(b(p), *args, None, F, 1 << 40, None) == -2
    assert lib.sale_cache_append(b(p), b(c), None, F, None) == -1 and lib.sale_cache_append(b(p), b(c), F, odd, None) == -2
    assert lib.sale_cache_append(b(p), None, F, F, None) == -1 and lib.sale_cache_append(None, b(c), F, F, None) == -1
    assert lib.sale_decode_attn(b(p), b(c), None, None, 0, F, None, F, 1 << 40, None) == -1
    assert lib.sale_decode_attn(b(p), b(c), F, None, 0, None, None, F, 1 << 40, None) == -1
    assert lib.sale_decode_attn(b(p), b(c), F, None, 5, F, None, F, 1 << 40, None) == -1      # a prefix without its pages
    assert lib.sale_decode_attn(b(p), b(c), F, F, -1, F, None, F, 1 << 40, None) == -2
    assert lib.sale_decode_attn(b(p), b(c), odd, None, 0, F, None, F, 1 << 40, None) == -2


def test_sizes_that_are_not_supported(sale):
    lib, c, b = sale.raw(), _cache(sale), ctypes.byref
    decode = lambda p, prefix=0: lib.sale_decode_attn(b(p), b(c), F, F, prefix, F, None, F, 1 << 40, None)
    assert decode(_params(sale, hq=64, hkv=1, n=2)) == -3             # 128 rows for one KV head
    assert decode(_params(sale, n=17)) == -3
    assert decode(_params(sale, batch=1, n=2, cu_seqlens=(0, 1, 2))) == -3
    assert decode(_params(sale), 1 << 30) == -3
    assert decode(_params(sale, batch=1 << 30)) == -3
    assert lib.sale_prompt_attn(b(_params(sale, batch=1, n=262145)), F, F, F, F, None, F, 1 << 60, None) == -3
    assert lib.sale_workspace_bytes(b(_params(sale, batch=1, n=262144)), sale.WS_PROMPT_ATTN) > 0
    assert lib.sale_prompt_attn(b(_params(sale, batch=1 << 20, n=262144)), F, F, F, F, None, F, 1 << 60, None) == -3


def test_launches_of_too_many_threads(sale):
    """2^24 workgroups of 256 threads and more."""
    lib, c, b = sale.raw(), _cache(sale), ctypes.byref
    append = lambda p: lib.sale_cache_append(b(p), b(c), F, F, None)
    assert append(_params(sale, batch=1, hq=32, hkv=32, n=1 << 24)) == -3      # a workgroup per token
    assert append(_params(sale, batch=1 << 24, hq=32, hkv=32, n=1)) == -3
    assert append(_params(sale, batch=1, hq=32, hkv=32, n=1 << 24, cu_seqlens=(0, 5, 1 << 24))) == -3
    big = (1 << 31) - 1
    for kw in (dict(batch=1 << 12, n=1 << 17), dict(batch=big, hq=big, hkv=big, n=64), dict(batch=big, hq=1, hkv=1, n=big)):
        assert lib.sale_workspace_bytes(b(_params(sale, **kw)), sale.WS_PROMPT_ATTN) == 0
        assert lib.sale_prompt_attn(b(_params(sale, **kw)), F, F, F, F, None, F, 1 << 60, None) == -3


def test_workspaces(sale):
    lib, c, b = sale.raw(), _cache(sale), ctypes.byref
    p = _params(sale, n=100)
    need = lib.sale_workspace_bytes(b(p), sale.WS_PROMPT_ATTN)
    assert need >= 2 * 2 * 2 * 128 * 256      # K' and V' of two batch entries, two heads, two blocks
    for ws, size in ((None, need), (F, need - 1), (ctypes.c_void_p(0x1008), need)):
        assert lib.sale_prompt_attn(b(p), F, F, F, F, None, ws, size, None) == -4
    p = _params(sale)
    need = lib.sale_decode_workspace_bytes(b(p), b(c), 40)
    assert need > 0 and lib.sale_decode_workspace_bytes(b(p), b(c), 0) < need
    for ws, size in ((None, need), (F, need - 1), (ctypes.c_void_p(0x1008), need)):
        assert lib.sale_decode_attn(b(p), b(c), F, F, 40, F, None, ws, size, None) == -4


@pytest.mark.parametrize("src,dst", [([0], [0]), ([0, 1], [2, 2]), ([0, 1], [1, 2]), ([0, 1], [2, 0]), ([10], [1]), ([1], [10]),
                                     ([-1], [1]), ([1], [-1]), ([0, 0, 0], [1, 2, 1])])
def test_copies_that_overlap(sale, src, dst):
    lib, p, c, b = sale.raw(), _params(sale), _cache(sale, table=None, lens=None), ctypes.byref
    i32 = ctypes.c_int32 * len(src)
    assert lib.sale_cache_copy(b(p), b(c), i32(*src), i32(*dst), len(src), None) == -2


def test_copies(sale):
    lib, p, c, b = sale.raw(), _params(sale), _cache(sale), ctypes.byref
    one = (ctypes.c_int32 * 1)(1)
    assert lib.sale_cache_copy(b(p), b(c), None, None, 0, None) == 0      # nothing to do, nothing launched
    assert lib.sale_cache_copy(b(p), b(c), None, one, 1, None) == -1
    assert lib.sale_cache_copy(b(p), b(c), one, one, -1, None) == -2
    assert lib.sale_cache_copy(b(_params(sale, head_dim=64)), b(c), one, one, 1, None) == -3
    assert lib.sale_cache_copy(b(_params(sale, hq=1 << 30, hkv=1 << 30)), b(_cache(sale, page_tokens=256)), one, (ctypes.c_int32 * 1)(2), 1, None) == -3


def test_the_binding_takes_device_tensors_only(sale):
    k = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        sale.Cache(k, k, torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="device tensor"):
        sale.prompt_attn(sale.Params(1, 2, 2, 5), *(torch.zeros(1, 2, 5, 128, dtype=torch.bfloat16) for _ in range(3)))


def test_prompts_of_nearly_2_31_tokens(sale):
    """Longer than any that is taken, also where their length and a block's would leave 32 bits together."""
    lib, b = sale.raw(), ctypes.byref
    for n in ((1 << 31) - 1, (1 << 31) - 63, (1 << 31) - 64, 1 << 30):
        for kw in (dict(batch=1, n=n), dict(batch=1, hq=1, hkv=1, n=n), dict(batch=1, n=n, cu_seqlens=(0, n)), dict(batch=1, n=n, cu_seqlens=(0, 0, n, n))):
            assert lib.sale_workspace_bytes(b(_params(sale, **kw)), sale.WS_PROMPT_ATTN) == 0
            assert lib.sale_prompt_attn(b(_params(sale, **kw)), F, F, F, F, None, F, (1 << 64) - 1, None) == -3


def test_joins_of_too_many_threads(sale):
    """More than 16 rows per KV head are joined 16 at a time, by workgroups of 512 threads: fewer than 2^32 of these too."""
    lib, b = sale.raw(), ctypes.byref
    c = _cache(sale, table_width=100)
    size = lambda prefix=0, **kw: lib.sale_decode_workspace_bytes(b(_params(sale, **kw)), b(c), prefix)
    call = lambda prefix=0, **kw: lib.sale_decode_attn(b(_params(sale, **kw)), b(c), F, F, prefix, F, None, F, 1 << 62, None)
    for kw in (dict(batch=(1 << 22) + 1, hq=17, hkv=1), dict(batch=1 << 22, hq=17, hkv=1), dict(batch=1 << 21, hq=49, hkv=1), dict(batch=1 << 20, hq=8, hkv=4, n=25),
               dict(batch=1 << 22, hq=1, hkv=1, n=33)):
        assert size(**kw) == 0 and call(**kw) == -3
        assert size(prefix=5, **kw) == 0 and call(prefix=5, **kw) == -3
    # (smaller by a sequence: taken)
    for kw in (dict(batch=(1 << 22) - 1, hq=17, hkv=1), dict(batch=(1 << 21) - 1, hq=49, hkv=1), dict(batch=(1 << 23) - 1, hq=1, hkv=1)):
        assert size(**kw) > 0
    # (left whole: there is no join)
    c = _cache(sale, table_width=4)
    assert lib.sale_decode_attn(b(_params(sale, batch=1 << 22, hq=17, hkv=1)), b(c), ctypes.c_void_p(0x1004), None, 0, F, None, None, 0, None) == -2
    assert call(prefix=5, batch=1 << 22, hq=17, hkv=1) == -3


class _Given:
    """What decode_workspace_bytes reads of a cache, without its tensors."""

    def __init__(self, c, kind="bf16"):
        self._struct, self._c = (c, 2, 128, 2, 0, (kind, c.page_tokens, c.table_width)), c

    def _arg(self, p, sequences=None):
        return self._c


def test_the_size_of_a_refused_cache_is_not_kept(sale):
    """Parameters keep the sizes that the library said for them; the 0 bytes of a cache that it refuses are none."""
    good = _cache(sale, table_width=100)
    need = sale.decode_workspace_bytes(sale.Params(2, 8, 2, 1), _Given(good))
    assert need > 0
    for bad in (_cache(sale, table_width=100, k_stride=(4224, 2112, 132)), _cache(sale, table_width=100, k=0x1008)):
        p = sale.Params(2, 8, 2, 1)
        assert sale.decode_workspace_bytes(p, _Given(bad)) == 0
        assert sale.decode_workspace_bytes(p, _Given(good)) == need
    assert sale.decode_workspace_bytes(p, _Given(_cache(sale, table_width=4))) == 0      # (needs none)


def test_parameters_keep_few_sizes(sale):
    """However many lengths of a prefix a program goes through."""
    p, c = sale.Params(2, 8, 2, 1), _Given(_cache(sale, table_width=100))
    attn = sale.workspace_bytes(p, sale.WS_PROMPT_ATTN)
    sizes = [sale.decode_workspace_bytes(p, c, n) for n in range(1, 3000)]
    assert len(p._ws_bytes) <= 300
    assert sale.workspace_bytes(p, sale.WS_PROMPT_ATTN) == attn and [sale.decode_workspace_bytes(p, c, n) for n in (1, 130, 2999)] == [sizes[i] for i in (0, 129, 2998)]


@pytest.mark.parametrize("pages", [[1.7], [0, 2.0], torch.zeros(2), torch.zeros(2, dtype=torch.int64), torch.zeros(1, 2, dtype=torch.int32),
                                   torch.zeros(4, dtype=torch.int32)[::2], [[1, 2]], [1 << 31], [-(1 << 31) - 1]])
def test_pages_that_are_no_list_of_pages(sale, pages):
    with pytest.raises(ValueError, match="src"):
        sale._host_pages("src", pages)


def test_lists_of_pages(sale):
    import numpy as np
    for pages in ([], [3, 1, (1 << 31) - 1], (5,), np.array([4, 2]), [np.int64(7)], torch.tensor([1, 2], dtype=torch.int32)):
        got = sale._host_pages("src", pages)
        assert got.dtype == torch.int32 and got.is_contiguous() and got.tolist() == [int(x) for x in pages]
