"""Host-side checks of the rotary and 8-bit-cache calls: frequencies, sizes, views, and what is refused before any launch."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import rotary
import paper_2510_26527_amd as psd
from paper_2510_26527_amd import runtime

P = [0x100000 + 0x10000 * i for i in range(12)]               # addresses nothing reads


def _rope(**kw):
    base = dict(d_head=64, rot_dim=0, layout=0, scaling=0, theta=1e4, factor=1.0, low=1.0, high=4.0, original_len=4096, magnitude=0.0)
    base.update(kw)
    return psd.psd_rope_create(psd.psd_rope_desc(**base))


def _model(**kw):
    base = dict(n_layers=2, d_model=128, n_q_heads=4, n_kv_heads=2, d_head=64, d_ffn=256, vocab=512, rope_theta=1e4, rms_eps=1e-5,
                dtype=psd.PSD_BF16)
    base.update(kw)
    d = psd.psd_model_desc(**base)
    return psd.psd_model_create(d, [0x1000] * (3 + 9 * d.n_layers))


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
@pytest.mark.parametrize("d,rot", [(64, 0), (128, 32), (80, 80), (256, 256), (2, 2), (6, 4)])
def test_frequencies(scaling, d, rot):
    code = {"none": 0, "linear": 1, "base": 2, "parts": 3}[scaling]
    r = _rope(d_head=d, rot_dim=rot, scaling=code, theta=5e5, factor=8.0, original_len=2048)
    n = (rot or d) // 2
    want = rotary.frequencies(rot or d, 5e5, scaling, 8.0, 1.0, 4.0, 2048)
    assert np.allclose(psd.psd_rope_frequencies(r, n), want, rtol=1e-12)
    psd.psd_rope_destroy(r)


@pytest.mark.parametrize("bad", [dict(d_head=0), dict(d_head=63), dict(d_head=258), dict(rot_dim=66), dict(rot_dim=7), dict(rot_dim=-2),
                                 dict(layout=2), dict(layout=-1), dict(scaling=4), dict(scaling=-1), dict(theta=0.0), dict(theta=float("inf")),
                                 dict(theta=float("nan")), dict(scaling=1, factor=0.0), dict(scaling=2, factor=float("nan")),
                                 dict(scaling=3, low=4.0), dict(scaling=3, low=-1.0), dict(scaling=3, original_len=0),
                                 dict(scaling=3, high=float("inf")), dict(magnitude=-1.0), dict(magnitude=float("inf"))])
def test_rope_refusals(bad):
    with pytest.raises(psd.PsdError) as e:
        _rope(**bad)
    assert e.value.status == psd.PSD_ERR_SHAPE


def test_rope_rotate_refusals():
    L, r = psd.lib(), _rope()
    call = lambda **kw: L.psd_rope_rotate(*{**dict(rope=r, x=P[0], y=P[1], pos=P[2], rows=3, heads=2, dtype=0, xs=128, ys=128, st=None), **kw}.values())
    assert call(rope=None) == psd.PSD_ERR_NULL and call(x=None) == psd.PSD_ERR_NULL and call(pos=None) == psd.PSD_ERR_NULL
    assert call(dtype=2) == psd.PSD_ERR_DTYPE
    for kw in (dict(rows=-1), dict(rows=(1 << 23) + 1), dict(heads=0), dict(heads=65536), dict(xs=127), dict(ys=0), dict(y=P[0], ys=256), dict(x=P[0] + 2), dict(pos=P[2] + 1)):
        assert call(**kw) == psd.PSD_ERR_SHAPE, kw
    assert call(rows=0, x=None, y=None, pos=None) == psd.PSD_OK
    psd.psd_rope_destroy(r)
    assert L.psd_rope_destroy(None) == psd.PSD_ERR_NULL and L.psd_rope_create(None, None) == psd.PSD_ERR_NULL


def test_model_set_rope():
    L, m, r = psd.lib(), _model(), _rope()
    other = _rope(d_head=128)
    assert L.psd_model_set_rope(None, r) == psd.PSD_ERR_NULL and L.psd_model_set_rope(m, other) == psd.PSD_ERR_SHAPE
    before = psd.psd_model_workspace_bytes(m, 1, 9, 256)
    assert L.psd_model_set_rope(m, r) == psd.PSD_OK
    psd.psd_rope_destroy(r)                                  # the model has its own copy
    assert psd.psd_model_workspace_bytes(m, 1, 9, 256) > 0
    assert L.psd_model_set_rope(m, None) == psd.PSD_OK and psd.psd_model_workspace_bytes(m, 1, 9, 256) == before
    psd.psd_rope_destroy(other)
    psd.psd_model_destroy(m)


def test_8_bit_cache_handles():
    L, m = psd.lib(), _model()
    assert psd.psd_kv_q8_bytes(m, 3, 192) == 2 * 3 * 2 * 192 * 64 and psd.psd_kv_q8_scale_bytes(m, 3, 192) == 2 * 3 * 2 * 3 * 4
    assert psd.psd_kv_q8_bytes(m, 3, 100) == 0 == psd.psd_kv_q8_scale_bytes(m, 0, 64)
    f32 = _model(dtype=psd.PSD_F32)
    assert psd.psd_kv_q8_bytes(f32, 1, 64) == 0
    out = ctypes.c_void_p()
    call = lambda **kw: L.psd_kv_create_q8(*{**dict(m=m, b=3, n=192, k=P[0], v=P[1], ks=P[2], vs=P[3], lens=P[4], ub=0, out=ctypes.byref(out)), **kw}.values())
    for kw in (dict(m=None), dict(k=None), dict(v=None), dict(ks=None), dict(vs=None), dict(lens=None), dict(out=None)):
        assert call(**kw) == psd.PSD_ERR_NULL, kw
    assert call(m=f32) == psd.PSD_ERR_DTYPE
    for kw in (dict(b=0), dict(n=100), dict(k=P[0] + 16), dict(vs=P[3] + 4)):
        assert call(**kw) == psd.PSD_ERR_SHAPE, kw
    assert call(ub=193) == psd.PSD_ERR_CAPACITY and call() == psd.PSD_OK
    view = psd.psd_kv8_layer(out, 1)
    assert (view.k_codes, view.v_codes) == (P[0] + 3 * 2 * 192 * 64, P[1] + 3 * 2 * 192 * 64)
    assert (view.k_scale, view.v_scale, view.lens) == (P[2] + 3 * 2 * 3 * 4, P[3] + 3 * 2 * 3 * 4, P[4])
    assert (view.batch, view.n_kv_heads, view.d_head, view.max_len) == (3, 2, 64, 192)
    assert L.psd_kv8_layer(out, 2, ctypes.byref(view)) == psd.PSD_ERR_SHAPE and L.psd_kv8_layer(None, 0, ctypes.byref(view)) == psd.PSD_ERR_NULL
    # token trees need the model's own type
    assert L.psd_model_forward_tree(m, P[5], 1, (ctypes.c_int32 * 1)(-1), out, P[6], P[7], 1 << 30, None) == psd.PSD_ERR_UNIMPLEMENTED
    assert L.psd_kv_compact_tree(out, P[5], P[6], P[7], 4, 2, -1, None) == psd.PSD_ERR_UNIMPLEMENTED
    plain = psd.psd_kv_create(m, 1, 64, _T(P[8]), _T(P[9]), _T(P[10]), 0)
    assert L.psd_kv8_layer(plain, 0, ctypes.byref(view)) == psd.PSD_ERR_DTYPE
    for kv in (out, plain):
        psd.psd_kv_destroy(kv)
    for x in (m, f32):
        psd.psd_model_destroy(x)


class _T:
    """Stands in for a tensor where the binding asks for its address."""

    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


def _view(**kw):
    base = dict(k_codes=P[0], v_codes=P[1], k_scale=P[2], v_scale=P[3], lens=P[4], batch=2, n_kv_heads=2, d_head=64, max_len=128)
    base.update(kw)
    return psd.psd_kv8_view(*base.values())


VIEW_REFUSALS = [(dict(k_codes=None), psd.PSD_ERR_NULL), (dict(v_scale=None), psd.PSD_ERR_NULL), (dict(lens=None), psd.PSD_ERR_NULL),
                 (dict(d_head=32), psd.PSD_ERR_SHAPE), (dict(batch=0), psd.PSD_ERR_SHAPE), (dict(batch=40000), psd.PSD_ERR_SHAPE),
                 (dict(n_kv_heads=3), psd.PSD_ERR_SHAPE), (dict(max_len=100), psd.PSD_ERR_SHAPE), (dict(k_codes=P[0] + 8), psd.PSD_ERR_SHAPE),
                 (dict(v_scale=P[3] + 2), psd.PSD_ERR_SHAPE)]


def test_append_refusals():
    L, r = psd.lib(), _rope()

    def call(view=None, **kw):
        a = {**dict(rope=r, q=P[5], k=P[6], v=P[7], q_out=P[8], n=3, h=4, dtype=1, qs=256, ks=128, vs=128, os=256, ub=100, st=None), **kw}
        return L.psd_kv8_append(ctypes.byref(view or _view()), *a.values())

    for kw in (dict(k=None), dict(v=None), dict(q=None), dict(q_out=None)):
        assert call(**kw) == psd.PSD_ERR_NULL, kw
    assert call(dtype=3) == psd.PSD_ERR_DTYPE
    for kw in (dict(n=0), dict(n=-1), dict(n=1 << 20), dict(h=3), dict(h=0), dict(qs=255), dict(ks=127), dict(vs=0), dict(os=255),
               dict(k=P[6] + 1), dict(q_out=P[5], os=512)):
        assert call(**kw) == psd.PSD_ERR_SHAPE, kw
    assert call(ub=129) == psd.PSD_ERR_CAPACITY and call(ub=2) == psd.PSD_ERR_CAPACITY
    big = _view(batch=64, n_kv_heads=1023, max_len=1 << 15)   # more blocks than a launch has
    assert call(big, n=16384, h=1023, qs=1023 * 64, ks=1023 * 64, vs=1023 * 64, os=1023 * 64, ub=16384) == psd.PSD_ERR_SHAPE
    other = _rope(d_head=128)
    assert call(rope=other) == psd.PSD_ERR_SHAPE
    for kw, status in VIEW_REFUSALS:
        assert call(_view(**kw)) == status, kw
    for x in (r, other):
        psd.psd_rope_destroy(x)


def test_attention_refusals():
    L = psd.lib()
    need = psd.psd_kv8_attention_workspace_bytes(2, 3, 4, 2, 64, 4000)
    assert need > 0 and psd.psd_kv8_attention_workspace_bytes(2, 3, 5, 2, 64, 4000) == 0 == psd.psd_kv8_attention_workspace_bytes(0, 3, 4, 2, 64, 4000)

    def call(view=None, **kw):
        a = {**dict(q=P[5], out=P[8], n=3, h=4, scale=0.0, qs=256, os=256, ub=4000, ws=P[9], size=need, st=None), **kw}
        return L.psd_kv8_attention(ctypes.byref(view or _view(max_len=4096)), *a.values())

    assert call(q=None) == psd.PSD_ERR_NULL and call(out=None) == psd.PSD_ERR_NULL
    for kw in (dict(n=0), dict(h=5), dict(qs=255), dict(os=260), dict(qs=248), dict(q=P[5] + 2), dict(out=P[8] + 8),
               dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**kw) == psd.PSD_ERR_SHAPE, kw
    assert call(ub=4097) == psd.PSD_ERR_CAPACITY and call(ub=2) == psd.PSD_ERR_CAPACITY
    for kw in (dict(ws=None), dict(ws=P[9] + 128), dict(size=need - 1)):
        assert call(**kw) == psd.PSD_ERR_WORKSPACE, kw
    for kw, status in VIEW_REFUSALS:
        assert call(_view(**{"max_len": 4096, **kw})) == status, kw


@pytest.mark.parametrize("args", [(1, 2**31 - 1, 64, 32, 128, 4096), (2**31 - 1, 1, 8, 8, 128, 4096), (1, 9, 2**31 - 1, 1, 128, 4096), (1, 9, 32, 8, 96, 4096),
                                  (1, 9, 32, 8, 0, 4096), (1, 9, 32, 8, -128, 4096), (1, 9, 32, 8, 128, 2**31 - 1), (1, 9, 32, 8, 128, 0), (1, 1 << 20, 32, 8, 128, 1 << 21)])
def test_no_workspace_size_for_what_the_call_refuses(args):
    assert psd.psd_kv8_attention_workspace_bytes(*args) == 0


def test_attention_into_its_own_queries_is_refused():
    L = psd.lib()
    assert L.psd_kv8_attention(ctypes.byref(_view()), P[5], P[5], 3, 4, 0.0, 256, 256, 100, P[9], 1 << 20, None) == psd.PSD_ERR_SHAPE


def test_a_closed_rope_is_refused():
    """Its missing handle would mean that nothing turns."""
    rope = runtime.Rope(64)
    rope.frequencies()
    rope.close()
    rope.close()
    for use in (lambda: rope.handle, rope.frequencies):
        with pytest.raises(ValueError):
            use()


def test_an_attention_objects_workspace_stays_on_its_device(monkeypatch):
    """Tensors of another device than the last call's get a workspace there; the old one stays for graphs."""
    used = []

    def launch(view, q, out, n, h_q, scale, qs, os, bound, ws, stream):
        if ws is None:
            raise psd.PsdError(psd.PSD_ERR_WORKSPACE, "attention")
        used.append(ws.device)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)          # (what get_device() says of the host)
    monkeypatch.setattr(runtime, "_raw", lambda device: 0)
    monkeypatch.setattr(psd, "psd_kv8_attention", launch)
    layer = runtime.KV8Layer(torch.zeros(1, 2, 4096, 64, dtype=torch.uint8), torch.zeros(1, 2, 64, 64, 64, dtype=torch.uint8), torch.ones(1, 2, 64),
                             torch.ones(1, 2, 64), torch.zeros(1, dtype=torch.int32))
    attend = runtime.KV8Attention()
    q = torch.zeros(1, 3, 4, 64, dtype=torch.bfloat16)
    attend(layer, q)
    class Elsewhere:
        device = torch.device("meta")

        def get_device(self):
            return 3

    old = attend._ws = Elsewhere()
    attend(layer, q)
    assert [d.type for d in used] == ["cpu", "cpu"] and attend._outgrown[-1] is old
