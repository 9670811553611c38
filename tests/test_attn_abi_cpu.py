"""What rotary positions, the paged cache and the attention over it refuse, on the host, before anything is launched (CPU only)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2508_02317_amd import libmoe
    return libmoe


ONE, ODD = 16, 20                                      # non-null and aligned, and misaligned: never dereferenced, validation fails first


def desc(L, **kw):
    d = dict(dtype=L.MOE_BF16, pages=4, heads=2, page_size=16, dim=128, reserved=0, k=ONE, v=ONE, k_scales=None, v_scales=None, page_stride=2 * 16 * 128,
             scale_page_stride=0)
    if kw.get("dtype") == L.MOE_MX8:
        d.update(k_scales=ONE, v_scales=ONE, scale_page_stride=2 * 16 * 4)
    d.update(kw)
    return L.moe_kv_cache_t(**d)


def rope_args(**kw):
    a = dict(q=ONE, qt=256, qh=128, k=ONE, kt=128, kh=128, dtype=1, T=4, Hq=2, Hk=1, D=128, rot=128, pos=ONE, cos=ONE, sin=ONE, n_pos=8, inter=0, qo=ONE, qot=256,
             qoh=128, ko=ONE, kot=128, koh=128, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=2), "UNSUPPORTED"), (dict(D=12, rot=0), "UNSUPPORTED"), (dict(D=520), "UNSUPPORTED"), (dict(rot=24), "UNSUPPORTED"), (dict(rot=256), "INVALID_ARG"),
    (dict(rot=-16), "INVALID_ARG"), (dict(T=-1), "INVALID_ARG"), (dict(Hq=0, Hk=0), "INVALID_ARG"), (dict(Hq=-1), "INVALID_ARG"), (dict(q=None), "INVALID_ARG"),
    (dict(ko=None), "INVALID_ARG"), (dict(cos=None), "INVALID_ARG"), (dict(pos=None), "INVALID_ARG"), (dict(n_pos=0), "INVALID_ARG"), (dict(q=ODD), "INVALID_ARG"),
    (dict(sin=ODD), "INVALID_ARG"), (dict(qt=260), "INVALID_ARG"), (dict(koh=4), "INVALID_ARG")])
def test_rope_refuses(L, bad, status):
    for call, name in ((L.lib.moe_rope_fwd, "moe_rope_fwd"), (L.lib.moe_rope_bwd, "moe_rope_bwd")):
        assert call(*rope_args(**bad)) == getattr(L, "MOE_ERR_" + status)
        assert name in L.moe_last_error()
    assert L.lib.moe_rope_fwd(*rope_args(T=0)) == L.MOE_OK


def test_rope_table_refuses(L):
    t = L.lib.moe_rope_table
    assert t(ONE, -1, 64, 1.0, ONE, ONE, None) == L.MOE_ERR_INVALID_ARG
    assert t(ONE, 8, 0, 1.0, ONE, ONE, None) == L.MOE_ERR_INVALID_ARG
    assert t(None, 8, 64, 1.0, ONE, ONE, None) == L.MOE_ERR_INVALID_ARG
    assert t(ONE, 8, 64, 1.0, ODD, ONE, None) == L.MOE_ERR_INVALID_ARG
    assert t(None, 0, 64, 1.0, None, None, None) == L.MOE_OK


BAD_CACHES = [(dict(dtype=3), "UNSUPPORTED"), (dict(pages=0), "INVALID_ARG"), (dict(heads=-1), "INVALID_ARG"), (dict(heads=2000), "UNSUPPORTED"), (dict(page_size=24), "UNSUPPORTED"),
              (dict(page_size=8), "UNSUPPORTED"), (dict(page_size=8192), "UNSUPPORTED"), (dict(dim=96), "UNSUPPORTED"), (dict(dim=512), "UNSUPPORTED"),
              (dict(page_stride=2 * 16 * 128 - 8), "INVALID_ARG"), (dict(page_stride=2 * 16 * 128 + 4), "INVALID_ARG"), (dict(k=None), "INVALID_ARG"), (dict(v=ODD), "INVALID_ARG"),
              (dict(dtype=2, k_scales=None), "INVALID_ARG"), (dict(dtype=2, v_scales=ODD), "INVALID_ARG"), (dict(dtype=2, scale_page_stride=64), "INVALID_ARG"),
              (dict(dtype=2, scale_page_stride=136), "INVALID_ARG")]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(L, bad, status):
    d = desc(L, **bad)
    c = ctypes.addressof(d)
    for rc in (L.lib.moe_kv_cache_write(c, ONE, 256, 128, ONE, 256, 128, 4, ONE, None, 0, 0, 0, 0, None, None, None, 0, 0, None, 0, 0, None),
               L.lib.moe_kv_cache_read(c, ONE, 2, ONE, None, 1, 4, ONE, ONE, None),
               L.lib.moe_paged_attn_decode(ONE, 1024, 128, c, ONE, 2, ONE, 1, 8, 1.0, 0, ONE, None, ONE, 1 << 30, None)):
        assert rc == getattr(L, "MOE_ERR_" + status), (bad, L.moe_last_error())


def test_null_caches(L):
    assert L.lib.moe_kv_cache_read(None, ONE, 2, ONE, None, 1, 4, ONE, ONE, None) == L.MOE_ERR_INVALID_ARG


def test_write_refuses(L):
    d = desc(L)
    base = dict(c=ctypes.addressof(d), k=ONE, kt=256, kh=128, v=ONE, vt=256, vh=128, T=4, slots=ONE, q=ONE, qt=1024, qh=128, Hq=8, rot=128, pos=ONE, cos=ONE, sin=ONE, n_pos=8,
                inter=0, qo=ONE, qot=1024, qoh=128, stream=None)
    call = lambda **kw: L.lib.moe_kv_cache_write(*dict(base, **kw).values())
    for bad in (dict(T=-1), dict(slots=None), dict(k=None), dict(q=None), dict(qo=ODD), dict(Hq=-2), dict(cos=None), dict(n_pos=-1), dict(kt=257), dict(vh=12), dict(qot=4)):
        assert call(**bad) == L.MOE_ERR_INVALID_ARG, bad
    assert call(rot=40) == L.MOE_ERR_UNSUPPORTED
    assert call(T=0) == L.MOE_OK


def test_read_refuses(L):
    d = desc(L)
    base = dict(c=ctypes.addressof(d), table=ONE, mp=2, rs=ONE, first=None, B=1, rows=4, k=ONE, v=ONE, stream=None)
    call = lambda **kw: L.lib.moe_kv_cache_read(*dict(base, **kw).values())
    for bad in (dict(B=-1), dict(rows=-1), dict(mp=-1), dict(table=None), dict(rs=None), dict(k=None), dict(v=ODD)):
        assert call(**bad) == L.MOE_ERR_INVALID_ARG, bad
    assert call(rows=0) == L.MOE_OK and call(B=0) == L.MOE_OK


def test_attention_refuses(L):
    d = desc(L)
    base = dict(q=ONE, qb=1024, qh=128, c=ctypes.addressof(d), table=ONE, mp=2, lens=ONE, B=1, Hq=8, scale=1.0, window=0, out=ONE, lse=ONE, ws=ONE, n=1 << 30, stream=None)
    call = lambda **kw: L.lib.moe_paged_attn_decode(*dict(base, **kw).values())
    for bad in (dict(B=-1), dict(Hq=0), dict(Hq=7), dict(mp=-1), dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(lens=None), dict(out=ODD),
                dict(lse=ODD), dict(table=None), dict(qb=1020), dict(qh=4)):
        assert call(**bad) == L.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(ws=None), dict(n=16), dict(ws=ODD)):
        assert call(**bad) == L.MOE_ERR_WORKSPACE, bad
    assert call(mp=1 << 28) == L.MOE_ERR_UNSUPPORTED                 # 2^32 tokens
    assert call(B=1 << 22, mp=1 << 10) == L.MOE_ERR_UNSUPPORTED
    assert call(B=0) == L.MOE_OK
    need = L.lib.moe_paged_attn_decode_workspace_bytes
    assert need(1, 8, 2, 128, 16, 2) >= 256 and need(-1, 8, 2, 128, 16, 2) == 256
    assert need(64, 32, 4, 128, 64, 128) == need(64, 32, 4, 128, 64, 4096)      # bounded by the workgroups, not by the contexts


def test_the_binding_refuses_what_is_not_a_cache(L):
    import torch
    mk = lambda *s, t=torch.bfloat16: torch.empty(s, dtype=t)
    with pytest.raises(ValueError):
        L.moe_kv_cache(mk(2, 2, 16, 128), mk(2, 2, 16, 128))         # not on a device
    with pytest.raises(TypeError):
        L.moe_kv_cache(mk(2, 2, 16, 128, t=torch.float16), mk(2, 2, 16, 128))


@pytest.mark.parametrize("which", ["k", "v", "k_scales", "v_scales"])
@pytest.mark.parametrize("how", ["swapped", "grown", "emptied", "replaced"])
def test_a_view_whose_tensor_has_moved_is_refused(L, which, how):
    """Calls go to the memory that the view's tensors had when it was made; where one has other memory by now, they are refused."""
    import torch

    class OnDevice(torch.Tensor):                                    # memory of the host that says it is a device's: nothing is launched
        is_cuda = True

    mk = lambda *s: torch.zeros(s, dtype=torch.uint8).as_subclass(OnDevice)
    view = L.moe_kv_cache(mk(3, 1, 16, 64), mk(3, 1, 16, 64), mk(3, 1, 16, 2), mk(3, 1, 16, 2))
    k, pages, lens = torch.zeros(2, 1, 64, dtype=torch.bfloat16), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    out = (torch.zeros(2, 1, 64, dtype=torch.bfloat16),) * 2
    calls = (lambda: L.moe_kv_cache_write(view, k, k, lens.long()), lambda: L.moe_kv_cache_read(view, pages, lens, out=out),
             lambda: L.moe_paged_attn_decode(k, view, pages, lens, out=out[0], ws=torch.zeros(4096)))
    assert view.ref == ctypes.addressof(view.desc)
    for call in calls:
        with pytest.raises(Exception) as e:                          # these are not on a device, and are refused for that
            call()
        assert "moved" not in str(e.value)
    t = getattr(view, which)
    was = t.data_ptr()
    if how == "swapped":
        t.data = torch.ones_like(t)
    elif how == "grown":
        t.resize_(3 << 20)
    elif how == "emptied":
        t.untyped_storage().resize_(0)
    else:
        setattr(view, which, mk(*t.shape))
    assert getattr(view, which).data_ptr() != was
    for call in calls:
        with pytest.raises(ValueError, match="%s.* moved" % which):
            call()
