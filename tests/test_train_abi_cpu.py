"""What the norm, the rotation by several axes and the router's losses refuse, on the host, before anything is launched (CPU only)."""
import ctypes

import pytest
import torch

from tests.test_attn_abi_cpu import desc

ONE, ODD = 16, 20                                      # non-null and aligned, and misaligned: never dereferenced, validation fails first
AXES = ctypes.create_string_buffer(bytes([0] * 16 + [1] * 24 + [2] * 24), 64)


@pytest.fixture(scope="module")
def L():
    from paper_2508_02317_amd import libmoe
    return libmoe


def axes_args(**kw):
    a = dict(q=ONE, qt=256, qh=128, k=ONE, kt=128, kh=128, dtype=1, T=4, Hq=2, Hk=1, D=128, rot=128, pos=ONE, n_axes=3, pair_axis=ctypes.addressof(AXES), cos=ONE, sin=ONE, n_pos=8,
             inter=0, qo=ONE, qot=256, qoh=128, ko=ONE, kot=128, koh=128, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("bad,status", [
    (dict(n_axes=0), "INVALID_ARG"), (dict(n_axes=5), "INVALID_ARG"), (dict(n_axes=-1), "INVALID_ARG"), (dict(pair_axis=None), "INVALID_ARG"), (dict(n_axes=2), "INVALID_ARG"),
    (dict(dtype=2), "UNSUPPORTED"), (dict(D=520), "UNSUPPORTED"), (dict(rot=24), "UNSUPPORTED"), (dict(T=-1), "INVALID_ARG"), (dict(Hq=0, Hk=0), "INVALID_ARG"),
    (dict(q=None), "INVALID_ARG"), (dict(ko=None), "INVALID_ARG"), (dict(pos=None), "INVALID_ARG"), (dict(n_pos=0), "INVALID_ARG"), (dict(sin=ODD), "INVALID_ARG"),
    (dict(qt=260), "INVALID_ARG")])
def test_rope_axes_refuses(L, bad, status):
    for call, name in ((L.lib.moe_rope_axes_fwd, "moe_rope_axes_fwd"), (L.lib.moe_rope_axes_bwd, "moe_rope_axes_bwd")):
        assert call(*axes_args(**bad)) == getattr(L, "MOE_ERR_" + status)
        assert name in L.moe_last_error()
    assert L.lib.moe_rope_axes_fwd(*axes_args(T=0)) == L.MOE_OK


def test_cache_write_axes_refuses(L):
    d = desc(L)
    args = lambda **kw: list(dict(dict(cache=ctypes.addressof(d), k=ONE, kt=256, kh=128, v=ONE, vt=256, vh=128, T=4, slots=ONE, q=ONE, qt=256, qh=128, Hq=2, rot=128, pos=ONE, n_axes=3,
                                       pair_axis=ctypes.addressof(AXES), cos=ONE, sin=ONE, n_pos=8, inter=0, qo=ONE, qot=256, qoh=128, stream=None), **kw).values())
    for bad in (dict(cache=None), dict(n_axes=0), dict(n_axes=5), dict(n_axes=1), dict(pair_axis=None), dict(slots=None), dict(pos=None), dict(kt=260), dict(q=ODD)):
        assert L.lib.moe_kv_cache_write_axes(*args(**bad)) == L.MOE_ERR_INVALID_ARG, bad
        assert "kv_cache_write_axes" in L.moe_last_error()
    assert L.lib.moe_kv_cache_write_axes(*args(T=0)) == L.MOE_OK


def fwd_args(**kw):
    a = dict(x=ONE, xt=64, xh=0, res=ONE, rt=64, rh=0, dtype=1, T=4, H=1, D=64, rms=0, w=ONE, b=ONE, wdtype=0, eps=1e-6, sum=ONE, st=64, sh=0, y=ONE, yt=64, yh=0, mean=ONE, rstd=ONE,
             stream=None)
    a.update(kw)
    return list(a.values())


def bwd_args(**kw):
    a = dict(dy=ONE, dt=64, dh=0, x=ONE, xt=64, xh=0, dtype=1, T=4, H=1, D=64, mean=ONE, rstd=ONE, w=ONE, wdtype=0, add=ONE, at=64, ah=0, dx=ONE, dxt=64, dxh=0, dw=ONE, db=ONE, ws=ONE,
             ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=2), "UNSUPPORTED"), (dict(wdtype=3), "UNSUPPORTED"), (dict(D=12), "UNSUPPORTED"), (dict(D=16392), "UNSUPPORTED"), (dict(D=0), "INVALID_ARG"), (dict(H=0), "INVALID_ARG"),
    (dict(T=-1), "INVALID_ARG"), (dict(T=1 << 20, H=1 << 12), "UNSUPPORTED"), (dict(x=None), "INVALID_ARG"), (dict(x=ODD), "INVALID_ARG"), (dict(xt=68), "INVALID_ARG"),
    (dict(xh=4), "INVALID_ARG"), (dict(w=ODD), "INVALID_ARG")])
def test_norm_refuses(L, bad, status):
    assert L.lib.moe_norm_fwd(*fwd_args(**bad)) == getattr(L, "MOE_ERR_" + status), L.moe_last_error()
    assert L.lib.moe_norm_bwd(*bwd_args(**bad)) == getattr(L, "MOE_ERR_" + status), L.moe_last_error()


def test_norm_refuses_what_only_one_direction_has(L):
    for bad in (dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")), dict(sum=None), dict(res=None), dict(y=None), dict(b=ODD), dict(rt=4), dict(sh=2), dict(yt=2)):
        assert L.lib.moe_norm_fwd(*fwd_args(**bad)) == L.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(dy=None), dict(rstd=None), dict(dx=None), dict(dw=ODD), dict(db=ODD), dict(at=4), dict(dxt=4), dict(add=ODD)):
        assert L.lib.moe_norm_bwd(*bwd_args(**bad)) == L.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(ws=None), dict(ws=ODD), dict(ws_bytes=L.lib.moe_norm_bwd_workspace_bytes(4, 1, 64) - 1)):
        assert L.lib.moe_norm_bwd(*bwd_args(**bad)) == L.MOE_ERR_WORKSPACE, bad
    assert L.lib.moe_norm_fwd(*fwd_args(T=0)) == L.MOE_OK and L.lib.moe_norm_bwd(*bwd_args(T=0, dw=None, db=None, ws=None)) == L.MOE_OK
    assert L.lib.moe_norm_bwd(*bwd_args(T=0, ws=None)) == L.MOE_ERR_WORKSPACE         # zeros are wanted
    assert L.lib.moe_norm_bwd_workspace_bytes(-1, 1, 64) == 0 and L.lib.moe_norm_bwd_workspace_bytes(4, 0, 64) == 0


def test_balance_refuses(L):
    ODD = 18                                           # 4-byte alignment is all that is asked for
    fwd = lambda **kw: list(dict(dict(z=ONE, idx=ONE, valid=None, T=4, E=8, k=2, losses=ONE, counts=ONE, imp=ONE, lse=ONE, ws=ONE, ws_bytes=1 << 20, stream=None), **kw).values())
    bwd = lambda **kw: list(dict(dict(z=ONE, counts=ONE, lse=ONE, valid=None, T=4, E=8, k=2, a=1.0, b=1.0, dl=None, add=None, out=ONE, stream=None), **kw).values())
    for bad, status in ((dict(T=-1), "INVALID_ARG"), (dict(E=0), "INVALID_ARG"), (dict(k=0), "INVALID_ARG"), (dict(k=9), "INVALID_ARG"), (dict(E=1025), "UNSUPPORTED"),
                        (dict(E=128, k=65), "UNSUPPORTED"), (dict(T=1 << 30), "UNSUPPORTED"), (dict(z=None), "INVALID_ARG"), (dict(z=ODD), "INVALID_ARG"),
                        (dict(counts=None), "INVALID_ARG"), (dict(lse=None), "INVALID_ARG"), (dict(lse=ODD), "INVALID_ARG")):
        for call, args in ((L.lib.moe_balance_loss_fwd, fwd), (L.lib.moe_balance_loss_bwd, bwd)):
            assert call(*args(**bad)) == getattr(L, "MOE_ERR_" + status), (bad, L.moe_last_error())
    for bad in (dict(idx=None), dict(losses=None), dict(imp=None), dict(T=0, counts=None), dict(losses=ODD)):
        assert L.lib.moe_balance_loss_fwd(*fwd(**bad)) == L.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(ws=None), dict(ws=ODD), dict(ws_bytes=L.lib.moe_balance_loss_fwd_workspace_bytes(4, 8, 2) - 1)):
        assert L.lib.moe_balance_loss_fwd(*fwd(**bad)) == L.MOE_ERR_WORKSPACE, bad
    for bad in (dict(out=None), dict(add=ODD), dict(dl=ODD)):
        assert L.lib.moe_balance_loss_bwd(*bwd(**bad)) == L.MOE_ERR_INVALID_ARG, bad
    assert L.lib.moe_balance_loss_bwd(*bwd(T=0)) == L.MOE_OK
    assert L.lib.moe_balance_loss_fwd_workspace_bytes(-1, 8, 2) == 0 and L.lib.moe_balance_loss_fwd_workspace_bytes(4, 0, 2) == 0


@pytest.mark.parametrize("compiled", [True, False])
def test_host_tensors_are_refused_by_name(L, monkeypatch, compiled):
    if compiled and L._marshal is None:
        pytest.skip("_marshal.so is not built here")
    if not compiled:
        monkeypatch.setattr(L, "_marshal", None)
    monkeypatch.setattr(L, "_current_device", lambda: 0)
    monkeypatch.setattr(L, "_stream", lambda: 0)
    monkeypatch.setattr(L, "_where", lambda: (0, 0))
    x, v = torch.zeros(4, 64), torch.zeros(4)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        L.moe_norm_fwd(x)
    with pytest.raises(ValueError, match="must be a device tensor"):
        L.moe_norm_bwd(x, x, v)
    with pytest.raises(ValueError, match="q must be a device tensor"):
        L.moe_rope_axes_fwd(x.view(4, 1, 64), None, v, v, v, b"")
    with pytest.raises(ValueError, match="must be given"):
        L.moe_rope_axes_fwd(None, None, v, v, v, b"")
    with pytest.raises(ValueError, match="must be a device tensor"):
        L.moe_balance_loss_fwd(x, torch.zeros((4, 2), dtype=torch.int32))
    with pytest.raises(ValueError, match="logits must be a device tensor"):
        L.moe_balance_loss_bwd(x, torch.zeros(65, dtype=torch.int32), v, 2)
