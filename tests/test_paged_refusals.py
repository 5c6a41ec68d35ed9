"""What the entry points of positions and the paged cache refuse, through the C
ABI, before anything is launched (no GPU: the addresses are never touched)."""
import ctypes

import pytest

from paper_2609_11356_amd import dg

A, B, C, D = 0x10000000, 0x20000000, 0x30000000, 0x40000000   # 16-byte aligned, far apart


def rope_params(**f):
    p = dg.dg_rope_params()
    p.struct_size = ctypes.sizeof(p)
    for k, v in dict(dict(dim=64, rotary=64, pairing=0, n_axes=1), **f).items():
        setattr(p, k, v)
    return p


def rope_create(**f):
    h = ctypes.c_void_p()
    st = dg.lib().dg_rope_desc_create(ctypes.byref(rope_params(**f)), ctypes.byref(h))
    if st == dg.DG_OK:
        dg.lib().dg_rope_desc_destroy(h)
    return st


def test_rotation_fields():
    assert rope_create() == dg.DG_OK
    for bad in (dict(dim=63), dict(dim=0), dict(dim=514, rotary=64), dict(rotary=66), dict(rotary=31), dict(rotary=0),
                dict(pairing=2), dict(n_axes=0), dict(n_axes=5), dict(n_axes=2), dict(struct_size=8)):
        assert rope_create(**bad) == dg.DG_ERR_INVALID, bad
    with pytest.raises(dg.DgError):
        dg.RopeDesc(64, axes=[0] * 31 + [4])
    with pytest.raises(ValueError):
        dg.RopeDesc(64, axes=[0] * 31)
    assert dg.lib().dg_rope_desc_create(None, None) == dg.DG_ERR_INVALID


def rope(desc, dtype=1, X=A, xt=512, xh=64, Y=B, yt=512, yh=64, pos=C, cos=D, sin=D, rows=100, T=10, H=8, inverse=0):
    return dg.lib().dg_rope(desc, dtype, X, xt, xh, Y, yt, yh, pos, cos, sin, rows, T, H, inverse, None)


def test_rope_refusals():
    d = dg.RopeDesc(64)
    h = d.handle
    assert rope(None) == dg.DG_ERR_INVALID
    assert rope(h, T=0) == dg.DG_OK and rope(h, H=0) == dg.DG_OK
    assert rope(h, dtype=3) == dg.DG_ERR_INVALID
    assert rope(h, inverse=2) == dg.DG_ERR_INVALID
    for bad in (dict(T=-1), dict(H=-1), dict(T=1 << 31), dict(H=65536), dict(xt=-1), dict(yh=-64), dict(rows=-1)):
        assert rope(h, **bad) == dg.DG_ERR_SHAPE, bad
    for bad in (dict(X=None), dict(Y=None), dict(pos=None), dict(cos=None), dict(sin=None),
                dict(Y=A + 16), dict(Y=A, yt=1024), dict(yh=32), dict(yt=64), dict(yt=0)):
        assert rope(h, **bad) == dg.DG_ERR_INVALID, bad
    for bad in (dict(X=A + 1), dict(Y=B + 1), dict(pos=C + 2), dict(cos=D + 1), dict(dtype=0, X=A + 2)):
        assert rope(h, **bad) == dg.DG_ERR_ALIGN, bad


def cache(**f):
    c = dg.dg_kv_cache()
    c.struct_size = ctypes.sizeof(c)
    d = dict(dtype=1, K=A, V=B, pages=10, page=16, heads=2, dim=64, page_stride=2048, token_stride=128,
             head_stride=64, k_scale=1.0, v_scale=1.0)
    for k, v in dict(d, **f).items():
        setattr(c, k, v)
    return c


BAD_CACHES = [(dict(struct_size=8), 1), (dict(dtype=0), 1), (dict(dtype=4), 1), (dict(K=None), 1), (dict(V=None), 1),
              (dict(k_scale=0.5), 1), (dict(dtype=3, k_scale=0.0), 1), (dict(dtype=3, v_scale=float("nan")), 1),
              (dict(dtype=3, v_scale=float("inf")), 1), (dict(dtype=3, k_scale=-1.0), 1),
              (dict(pages=0), 3), (dict(pages=1 << 27), 3), (dict(page=0), 3), (dict(heads=0), 3), (dict(dim=0), 3), (dict(page_stride=-16), 3),
              (dict(K=A + 8), 4), (dict(V=B + 2), 4), (dict(token_stride=132), 4), (dict(head_stride=68), 4),
              (dict(page_stride=2052), 4), (dict(dtype=3, head_stride=72), 4)]


def append(desc, c, dtype=1, Q=C, Qout=D, qh=4, K=C, V=C, pos=C, cos=C, sin=C, rows=10, slots=C, T=5):
    return dg.lib().dg_kv_append(desc, ctypes.addressof(c) if c is not None else None, dtype, Q, 512, 64, Qout, 512,
                                 64, qh, K, 512, 64, V, 512, 64, pos, cos, sin, rows, slots, T, None)


def test_append_refusals():
    d = dg.RopeDesc(64)
    for fields, status in BAD_CACHES:
        assert append(d.handle, cache(**fields)) == status, fields
    assert append(d.handle, None) == dg.DG_ERR_INVALID
    c = cache()
    assert append(d.handle, c, T=0) == dg.DG_OK
    for bad in (dict(dtype=0), dict(dtype=3), dict(Qout=None), dict(Q=None), dict(K=None), dict(V=None),
                dict(slots=None), dict(pos=None), dict(cos=None), dict(Qout=C + 64)):
        assert append(d.handle, c, **bad) == dg.DG_ERR_INVALID, bad
    assert append(None, c) == dg.DG_ERR_INVALID                     # queries without a rotation
    assert append(d.handle, cache(V=A)) == dg.DG_ERR_INVALID        # K and V in one place
    assert append(d.handle, c, dtype=2) == dg.DG_ERR_UNSUPPORTED
    assert append(d.handle, cache(dtype=3), dtype=2) == dg.DG_ERR_UNSUPPORTED
    for bad in (dict(T=-1), dict(T=1 << 31), dict(qh=-1), dict(rows=-1)):
        assert append(d.handle, c, **bad) == dg.DG_ERR_SHAPE, bad
    assert append(d.handle, cache(dim=66, head_stride=72, token_stride=144)) == dg.DG_ERR_SHAPE
    for bad in (dict(K=C + 1), dict(slots=C + 4), dict(pos=C + 2), dict(Q=C + 1)):
        assert append(d.handle, c, **bad) == dg.DG_ERR_ALIGN, bad


def attend(d, c, dtype=1, Q=C, qt=512, qh=64, cu=C, kv=C, table=C, width=8, tstride=8, O=D, ot=512, oh=64, rows=20,
           heads=8, batch=3, max_q=9, max_kv=128, scale=0.1, ws=None, wb=0):
    return dg.lib().dg_attention_paged(d and d.handle, dtype, Q, qt, qh, ctypes.addressof(c) if c is not None else None,
                                       cu, kv, table, width, tstride, O, ot, oh, rows, heads, batch, max_q, max_kv,
                                       scale, ws, wb, None)


def test_attention_refusals():
    d, c = dg.AttnDesc(causal=1, split_keys=64), cache()
    assert attend(None, c) == dg.DG_ERR_INVALID and attend(d, None) == dg.DG_ERR_INVALID
    for fields, status in BAD_CACHES:
        assert attend(d, cache(**fields)) == status, fields
    for none in (dict(rows=0), dict(heads=0), dict(batch=0), dict(max_q=0)):
        assert attend(d, c, **none) == dg.DG_OK, none
    for desc in (dict(key_block=32), dict(key_block=128), dict(block_sum="seq"), dict(pv_fma=0), dict(p_dtype="f16"),
                 dict(causal=1, q_block=80)):
        assert attend(dg.AttnDesc(**desc), c) == dg.DG_ERR_UNSUPPORTED, desc
    assert attend(d, cache(dim=96, head_stride=96, token_stride=192)) == dg.DG_ERR_UNSUPPORTED
    assert attend(d, c, dtype=2) == dg.DG_ERR_UNSUPPORTED
    assert attend(d, cache(dtype=2)) == dg.DG_ERR_UNSUPPORTED        # bf16 probabilities over binary16
    for bad in (dict(rows=-1), dict(heads=7), dict(heads=-2), dict(batch=-1), dict(batch=65536), dict(max_q=-1),
                dict(max_kv=-1), dict(max_kv=(1 << 31) - 1), dict(width=-1), dict(width=1 << 28), dict(tstride=7),
                dict(qt=-1), dict(oh=-1), dict(rows=1 << 29), dict(rows=(1 << 25) + 1)):
        assert attend(d, c, **bad) == dg.DG_ERR_SHAPE, bad
    assert attend(d, cache(heads=300), heads=300, batch=60000) == dg.DG_ERR_SHAPE
    for wide in (dict(page_stride=1 << 30), dict(token_stride=1 << 27)):
        assert attend(d, cache(**wide)) == dg.DG_ERR_SHAPE, wide
    for bad in (dict(Q=None), dict(O=None), dict(cu=None), dict(kv=None), dict(table=None), dict(O=C), dict(ot=64),
                dict(oh=32)):
        assert attend(d, c, **bad) == dg.DG_ERR_INVALID, bad
    for bad in (dict(Q=C + 8), dict(O=D + 8), dict(qt=516), dict(oh=68), dict(cu=C + 2), dict(kv=C + 1), dict(table=C + 3)):
        assert attend(d, c, **bad) == dg.DG_ERR_ALIGN, bad
    assert attend(d, c, ws=A, wb=16) == dg.DG_ERR_SCRATCH
    need = dg.lib().dg_attention_paged_bytes(d.handle, ctypes.addressof(c), 20, 8, 3, 9, 128)
    assert need > 0 and attend(d, c, ws=A + 8, wb=need) == dg.DG_ERR_ALIGN
    inst = dg.AttnDesc(causal=1, exp2="inst")
    for scale in (0.0, -1.0, float("nan")):
        assert attend(inst, c, scale=scale) == dg.DG_ERR_INVALID
    # one span takes no workspace; a refused call none either
    assert dg.lib().dg_attention_paged_bytes(dg.AttnDesc().handle, ctypes.addressof(c), 20, 8, 3, 9, 128) == 0
    assert dg.lib().dg_attention_paged_bytes(d.handle, ctypes.addressof(c), 20, 7, 3, 9, 128) == 0


def test_descriptor_fields_of_the_paged_form():
    for bad in (dict(split_keys=-64), ):
        with pytest.raises(dg.DgError) as e:
            dg.AttnDesc(**bad)
        assert e.value.status == dg.DG_ERR_INVALID
    with pytest.raises(dg.DgError) as e:
        dg.AttnDesc(split_keys=96)
    assert e.value.status == dg.DG_ERR_UNSUPPORTED
    # dg_attention has none of them
    for only_paged in (dict(split_keys=64), dict(exp2="inst"), dict(p_dtype="f16"), dict(out="f16")):
        d = dg.AttnDesc(**only_paged)
        assert dg.lib().dg_attention(d.handle, A, B, C, D, 1, 4, 4, 64, 0.1, None) == dg.DG_ERR_UNSUPPORTED


def test_the_struct_before_the_paged_fields_is_taken():
    p = dg.dg_attn_params()
    p.struct_size = dg.dg_attn_params.split_keys.offset
    for k, v in dict(key_block=64, q_block=64, block_sum=2, p_dtype=1, pv_fma=1, out_dtype=1, split_keys=77,
                     exp2=9).items():
        setattr(p, k, v)     # what lies behind the given size is not read
    h = ctypes.c_void_p()
    assert dg.lib().dg_attn_desc_create(ctypes.byref(p), ctypes.byref(h)) == dg.DG_OK
    dg.lib().dg_attn_desc_destroy(h)
    for size in (p.struct_size - 4, p.struct_size + 4):
        p.struct_size = size
        assert dg.lib().dg_attn_desc_create(ctypes.byref(p), ctypes.byref(h)) == dg.DG_ERR_INVALID
