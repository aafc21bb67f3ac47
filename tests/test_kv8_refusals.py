"""Frequencies on the host, and what the rotary and 8-bit cache calls refuse before anything reaches a GPU (CPU only)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2505_08600_amd import api

L = api.lib()
GOOD = 1 << 20  # an aligned address that a refused call never touches


def cfg(**kw):
    d = dict(rot_dim=64, scaling=0, base=10000.0, factor=4.0, low=1.0, high=4.0, trained_len=4096.0)
    d.update(kw)
    return api._RopeConfig(*[d[n] for n, _ in api._RopeConfig._fields_])


def test_frequencies_of_every_scaling():
    R, base = 64, 10000.0
    i = np.arange(R // 2)
    f = base ** (-2.0 * i / R)
    close = lambda a, b: np.testing.assert_allclose(a, b, rtol=1e-14)
    close(api.rope_freqs(R), f)
    close(api.rope_freqs(R, "linear", factor=4.0), f / 4)
    turns = 4096 * f / (2 * math.pi)
    keep = np.clip((turns - 1) / 3, 0, 1)
    got = api.rope_freqs(R, "bands", factor=4.0, low=1.0, high=4.0, trained_len=4096.0)
    np.testing.assert_allclose(got, keep * f + (1 - keep) * f / 4, rtol=1e-12)
    assert (got[turns >= 4] == api.rope_freqs(R)[turns >= 4]).all() and np.allclose(got[turns <= 1], f[turns <= 1] / 4, rtol=1e-14)
    lo = math.floor(R * math.log(4096 / (2 * math.pi * 32)) / (2 * math.log(base)))
    hi = math.ceil(R * math.log(4096 / (2 * math.pi * 1)) / (2 * math.log(base)))
    g = np.clip((i - lo) / (hi - lo), 0, 1)
    got = api.rope_freqs(R, "ramp", factor=4.0, low=1.0, high=32.0, trained_len=4096.0)
    np.testing.assert_allclose(got, (1 - g) * f + g * f / 4, rtol=1e-12)
    assert (np.diff(got) < 0).all()
    assert len(api.rope_freqs(2)) == 1 and len(api.rope_freqs(512)) == 256


def test_refused_rotary_configurations():
    out = (C.c_double * 256)()
    ok = lambda c: L.sd_rope_freqs(C.byref(c), out)
    assert ok(cfg()) == api.SD_OK
    bad = [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=514), dict(scaling=4), dict(scaling=-1), dict(base=1.0),
           dict(base=math.nan), dict(base=math.inf), dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.nan),
           dict(scaling=2, low=0.0), dict(scaling=2, low=4.0), dict(scaling=3, trained_len=0.5),
           dict(scaling=3, trained_len=math.inf), dict(scaling=2, high=math.inf)]
    for kw in bad:
        assert ok(cfg(**kw)) == api.SD_EINVAL, kw
    assert ok(cfg(factor=0.0, low=0.0, trained_len=0.0)) == api.SD_OK        # not read by the plain frequencies
    assert L.sd_rope_freqs(None, out) == api.SD_EINVAL and L.sd_rope_freqs(C.byref(cfg()), None) == api.SD_EINVAL
    assert L.sd_model_set_rope(None, C.byref(cfg()), 1.0) == api.SD_EINVAL


def test_refused_rotations():
    def rope(x=GOOD, xr=64, xh=64, y=GOOD + 4096, yr=64, yh=64, dt=0, rows=1, heads=1, dim=64, rot=64, pos=GOOD, f=GOOD,
             gain=1.0, inter=0, inv=0):
        return L.sd_rope(x, xr, xh, y, yr, yh, dt, rows, heads, dim, rot, pos, f, gain, inter, inv, None)
    bad = [dict(x=None), dict(y=None), dict(pos=None), dict(f=None), dict(dt=2), dict(rows=0), dict(heads=0), dict(dim=1),
           dict(dim=514), dict(rot=0), dict(rot=63), dict(rot=66), dict(rows=2, xr=63), dict(heads=2, yh=32), dict(xr=-1),
           dict(rows=2, y=GOOD, yr=128), dict(gain=math.nan), dict(inter=2), dict(x=GOOD + 2), dict(f=GOOD + 4),
           dict(pos=GOOD + 2), dict(heads=1 << 20, xh=64, yh=64)]
    for kw in bad:
        assert rope(**kw) == api.SD_EINVAL, kw
        assert b"sd_rope" in L.sd_last_error()


def cache(**kw):
    d = dict(k=GOOD, v=GOOD, k_scale=GOOD, v_scale=GOOD, tokens=64, n_kv_heads=2, head_dim=64, n_seq=2, off=GOOD, cap=GOOD, status=None)
    d.update(kw)
    return api._Kv8(*[d[n] for n, _ in api._Kv8._fields_])


BAD_CACHES = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(off=None), dict(cap=None), dict(tokens=0),
              dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(head_dim=8), dict(head_dim=72), dict(head_dim=272), dict(n_seq=0),
              dict(k=GOOD + 8), dict(v=GOOD + 4), dict(v_scale=GOOD + 2), dict(off=GOOD + 4), dict(status=GOOD + 1)]


@pytest.mark.parametrize("name", ["sd_kv8_append", "sd_kv8_read"])
def test_refused_moves(name):
    def move(c=cache(), n_seq=2, length=GOOD, row_start=None, rows=4, dt=0, k=GOOD, kr=128, kh=64, v=GOOD, vr=128, vh=64):
        return getattr(L, name)(C.byref(c) if c is not None else None, None, n_seq, length, row_start, rows, dt, k, kr, kh, v, vr, vh, None)
    for kw in BAD_CACHES:
        assert move(c=cache(**kw)) == api.SD_EINVAL, kw
        assert name.encode() in L.sd_last_error()
    bad = [dict(c=None), dict(n_seq=0), dict(n_seq=3), dict(length=None), dict(rows=0), dict(rows=3), dict(rows=(1 << 23) + 1, row_start=GOOD),
           dict(dt=2), dict(kr=63), dict(kh=-1), dict(vh=32), dict(k=GOOD + 2), dict(v=GOOD + 1), dict(k=None, v=None)]
    bad += [dict(k=None), dict(v=None)] if name == "sd_kv8_append" else []
    for kw in bad:
        assert move(**kw) == api.SD_EINVAL, kw


def attn(**kw):
    d = dict(seq_ids=None, len=GOOD, row_start=None, n_seq=2, rows=4, max_rows=0, max_len=64, n_heads=4, dtype=1, q=GOOD, q_row=256,
             q_head=64, out=GOOD, o_row=256, o_head=64, lse=None, scale=0.125, causal=1, window=0, sinks=0, workspace=None, workspace_bytes=0)
    d.update(kw)
    return api._Kv8Attn(*[d[n] for n, _ in api._Kv8Attn._fields_])


def test_refused_attention():
    def go(c=cache(), a=attn()):
        return L.sd_kv8_attend(C.byref(c), C.byref(a) if a is not None else None, None)
    for kw in BAD_CACHES:
        assert go(c=cache(**kw)) == api.SD_EINVAL, kw
        assert L.sd_kv8_attend_workspace(C.byref(cache(**kw)), C.byref(attn())) == api.SD_EINVAL
    bad = [dict(len=None), dict(n_seq=0), dict(n_seq=3), dict(rows=0), dict(rows=5), dict(max_rows=-1), dict(max_len=-1), dict(n_heads=0),
           dict(n_heads=3), dict(dtype=2), dict(q=None), dict(out=None), dict(q=GOOD + 1), dict(out=GOOD + 1), dict(q_row=32),
           dict(o_head=32), dict(lse=GOOD + 2), dict(scale=math.nan), dict(scale=math.inf), dict(window=-1), dict(sinks=-1), dict(sinks=4),
           dict(window=8, causal=0)]
    for kw in bad:
        assert go(a=attn(**kw)) == api.SD_EINVAL, kw
        assert L.sd_kv8_attend_workspace(C.byref(cache()), C.byref(attn(**kw))) == api.SD_EINVAL, kw
    assert go(a=None) == api.SD_EINVAL
    assert go(a=attn(workspace=GOOD + 8, workspace_bytes=1 << 20)) == api.SD_EINVAL
    assert go(a=attn(workspace=GOOD, workspace_bytes=-1)) == api.SD_EINVAL
    assert L.sd_kv8_attend_workspace(C.byref(cache()), C.byref(attn())) >= 0


def test_scales_that_leave_the_range():
    assert L.sd_kv8_attend(C.byref(cache()), C.byref(attn(scale=3e38)), None) == api.SD_EINVAL   # times log2(e)
    assert L.sd_kv8_attend(C.byref(cache()), C.byref(attn(scale=-3e38)), None) == api.SD_EINVAL


@pytest.mark.parametrize("rows", [1 << 23, 4096, 2])
@pytest.mark.parametrize("max_rows", [0, 1, 2 ** 31 - 1])
@pytest.mark.parametrize("window", [0, 100, 2 ** 31 - 1])
def test_workspace_of_the_longest_contexts(rows, max_rows, window):
    """At most 128 parts of every row, whatever the lengths."""
    a = attn(rows=rows, row_start=GOOD, max_rows=max_rows, max_len=2 ** 31 - 1, window=window)
    need = L.sd_kv8_attend_workspace(C.byref(cache(tokens=2 ** 40)), C.byref(a))
    one = rows * 4 * (64 + 4) * 4
    assert 0 <= need <= 128 * one and need % one == 0


def test_refused_contexts():
    assert L.sd_ctx_attach_kv8(None, None, 0, 0) == api.SD_EINVAL
    assert L.sd_ctx_get_kv(None, None, 0, 0, None, None, 1) == api.SD_EINVAL


def test_binding_refuses_what_does_not_fit():
    import torch
    x = torch.zeros(2, 3, 64)
    with pytest.raises(ValueError):
        api.sd_rope(x, torch.zeros(2, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))     # not on a GPU
    with pytest.raises(ValueError):
        api.sd_rope(x.half(), torch.zeros(2, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        api.Kv8Cache(torch.zeros(1, 4, 64, dtype=torch.int8), *(None,) * 5)
    with pytest.raises(KeyError):
        api.rope_freqs(64, "other")
