"""What the Python binding does around the library's calls: shapes that the library refuses arrive there, a cache's words are shown where they lie."""
import types

import pytest

SHAPES = [(4, 1024), (2048, 2), (3, 2048), (4096, 1), (1 << 20, 4), (4, 0), (0, 16), (-3, 16), (4, -16), (4, 24)]


@pytest.mark.parametrize("heads,dim", SHAPES)
@pytest.mark.parametrize("max_tokens", [None, 8, 0, -1])
def test_a_cache_of_any_shape_is_refused_by_the_library(heads, dim, max_tokens):
    """Without a context every creation is refused; what is computed from the shape must not end before that."""
    from paper_2602_11470_amd import binding as B
    with pytest.raises(B.CachemirError) as e:
        B.KvCache(types.SimpleNamespace(S=2048, h=None), heads, dim, 0, 3, 0.0, max_tokens)
    assert e.value.status == -1


def test_words_are_asked_for_on_the_device_of_the_context(monkeypatch):
    """The memory lies on the context's device; asked for on the current one, another device would silently get a copy."""
    import torch
    from paper_2602_11470_amd import binding as B
    asked = []

    def as_tensor(words, device=None):
        asked.append(torch.device(device))
        return torch.zeros(words.__cuda_array_interface__["shape"], dtype=torch.int64)
    monkeypatch.setattr(B.lib, "cm_kv_view", lambda *a: 0)
    monkeypatch.setattr(B.torch, "as_tensor", as_tensor)
    kv = B.KvCache.__new__(B.KvCache)
    kv.ctx, kv.h, kv.level, kv.dim, kv.r_i, kv.pages = types.SimpleNamespace(n=8, device=torch.device("cuda", 3)), None, 2, 4, 2, 3
    kv._words, kv._owner = {}, None
    assert kv.words(B.CM_QK).shape == (3, 2, 3, 8) and kv.words(B.CM_SV).shape == (4, 2, 3, 8) and kv.words(B.CM_KV_INDEX).shape == (2, 2, 2, 3, 8)
    assert asked == [torch.device("cuda", 3)] * 3


@pytest.mark.gpu
def test_words_lie_where_the_library_says():
    import ctypes as C
    import torch
    from paper_2602_11470_amd import binding as B
    ctx = B.config1()
    try:
        kv = ctx.kv_create(4, 16, 3, key_index=True)
        assert ctx.device == torch.device("cuda", torch.cuda.current_device())
        for which in (B.CM_QK, B.CM_SV, B.CM_KV_INDEX):
            d = B.cm_ct()
            assert B.lib.cm_kv_view(kv.h, which, 0, C.byref(d)) == 0
            assert kv.words(which).data_ptr() == d.dev and kv.words(which).device == ctx.device
    finally:
        ctx.close()


@pytest.mark.gpu
def test_shapes_that_do_not_fit_say_so():
    from paper_2602_11470_amd import binding as B
    ctx = B.config1()
    try:
        for heads, dim, status in ((4, 1024, -5), (2048, 2, -5), (3, 2048, -5), (4, 24, -5), (4, 0, -1), (0, 16, -1), (4, -16, -1)):
            with pytest.raises(B.CachemirError) as e:
                ctx.kv_create(heads, dim, 3, max_tokens=8)
            assert e.value.status == status
            with pytest.raises(B.CachemirError) as e:
                ctx.kv_create(heads, dim, 3)
            assert e.value.status in (-1, -5)
        assert ctx.kv_create(4, 16, 3).pages == 16 and ctx.kv_create(4, 16, 3, max_tokens=33).pages == 2
    finally:
        ctx.close()


@pytest.mark.gpu
def test_head_counts_whose_product_with_the_dims_passes_32_bits():
    import ctypes as C
    from paper_2602_11470_amd import binding as B
    ctx = B.config1()
    try:
        h = C.c_void_p()
        for heads, dim in ((1 << 20, 1 << 12), (1 << 16, 1 << 16), (1 << 30, 4), ((1 << 31) - 1, 2), (2, 1 << 30)):
            assert B.lib.cm_kv_create_ex(ctx.h, heads, dim, 0, 3, 0.0, 8, 0, C.byref(h)) == -5
            assert B.lib.cm_rope_create(ctx.h, heads, dim, 3, 0, 0, 10000.0, None, C.byref(h)) == -5
        assert h.value is None
    finally:
        ctx.close()
