"""More of what positions and the paged cache refuse or reserve, through the C ABI,
before anything is launched (no GPU: the addresses are never touched)."""
import ctypes

from paper_2609_11356_amd import dg
from tests.test_paged_refusals import A, B, C, D, append, attend, cache, rope  # noqa: F401


def test_strides_whose_offsets_pass_63_bits():
    """Each stride below 2^40 and each count below 2^31, but not their products."""
    r = dg.RopeDesc(64)
    h = r.handle
    far = 1 << 39
    for bad in (dict(T=(1 << 31) - 1, xt=far, yt=far), dict(T=(1 << 31) - 1, xt=far), dict(T=(1 << 31) - 1, yt=far),
                dict(dtype=0, T=1 << 25, yt=far)):
        assert rope(h, **dict(dict(X=A, Y=B), **bad)) == dg.DG_ERR_SHAPE, bad
    wide = cache(pages=1 << 27, page=8, page_stride=far)
    assert append(h, wide) == dg.DG_ERR_SHAPE
    d, c = dg.AttnDesc(causal=1, split_keys=64), cache()
    far_append = lambda Q=None, Qout=None, q=512, qo=512, k=512, v=512: dg.lib().dg_kv_append(   # noqa: E731
        h, ctypes.addressof(c), 1, Q, q, 64, Qout, qo, 64, 4, C, k, 64, C, v, 64, C, C, C, 10, C, 1 << 27, None)
    for bad in (dict(Q=C, Qout=D, q=far), dict(Q=C, Qout=D, qo=far), dict(k=far), dict(v=far)):
        assert far_append(**bad) == dg.DG_ERR_SHAPE, bad
    for bad in (dict(qt=far, rows=1 << 24), dict(ot=far, rows=1 << 24)):
        assert attend(d, c, **bad) == dg.DG_ERR_SHAPE, bad


def test_scales_whose_product_is_not_above_zero():
    """The part's exponential takes qk_scale * k_scale in binary32, which has to stay above 0:
    0 times the -inf of a key that is not seen would be NaN."""
    inst, lib = (dg.AttnDesc(causal=1, exp2=e) for e in ("inst", "lib"))
    small = cache(dtype=3, k_scale=1e-30)
    assert attend(inst, small, scale=1e-30, rows=0) == dg.DG_ERR_INVALID
    assert attend(inst, small, scale=1e-3, rows=0) == dg.DG_OK
    assert attend(lib, small, scale=1e-30, rows=0) == dg.DG_OK


def test_views_of_one_tensor_that_share_elements():
    """At the same strides rows may lie between each other, but not less than a head apart."""
    r = dg.RopeDesc(64)
    h = r.handle
    for shift in (1, 63, 64, 64 * 7, 512 - 63, 512, 512 * 9 + 63):
        for sign in (1, -1):
            assert rope(h, X=B, Y=B + sign * 2 * shift) == dg.DG_ERR_INVALID, shift
    # between the rows, but for one element; at other strides
    for bad in (dict(xt=1024, yt=1024, Y=A + 2 * (512 - 63)), dict(xt=1024, yt=1024, xh=128, yh=128, Y=A + 2 * 63),
                dict(xt=1024, yt=2048, Y=A + 2 * 512), dict(xt=1024, yt=1024, xh=64, yh=128, Y=A + 2 * 512)):
        assert rope(h, X=A, **bad) == dg.DG_ERR_INVALID, bad


def test_append_to_rows_that_share_memory():
    """Attention reads a cache whose heads or pages are one and the same; an append would leave
    there what came last."""
    r, d = dg.RopeDesc(64), dg.AttnDesc(causal=1)
    h = r.handle
    for shared in (dict(head_stride=0), dict(token_stride=0), dict(page_stride=0), dict(head_stride=32),
                   dict(token_stride=64, head_stride=64), dict(page_stride=1920), dict(page_stride=64, token_stride=640)):
        assert append(h, cache(**shared)) == dg.DG_ERR_INVALID, shared
        assert attend(d, cache(**shared), rows=0) == dg.DG_OK, shared
    # of one head, token or page the stride does not count; any order of the three
    for fine in (dict(heads=1, head_stride=0), dict(pages=1, page_stride=0), dict(page=1, token_stride=0),
                 dict(token_stride=64, head_stride=1024), dict(page_stride=128, token_stride=1280)):
        assert append(h, cache(**fine), T=0) == dg.DG_OK, fine


def space(d, c, rows, q_heads, batch, max_q, max_kv):
    return dg.lib().dg_attention_paged_bytes(d.handle, ctypes.addressof(c), rows, q_heads, batch, max_q, max_kv)


def test_records_are_of_rows_that_there_may_be():
    d, each = dg.AttnDesc(causal=1, split_keys=512), (64 + 2) * 4 * 8      # 8 spans
    one = cache(heads=1)
    # 32 query heads over 1: no sequence has 1 to 16 rows
    assert space(d, one, 64, 32, 64, 1, 4096) == 64 * 32 * each
    # 3 over 1, up to 3 tokens: 9 rows each
    assert space(d, one, 64, 3, 64, 3, 4096) == 64 * 9 * each
    # tokens one at a time: no row too many
    assert space(d, cache(heads=8, page_stride=8192, token_stride=512), 64, 32, 64, 1, 4096) == 64 * 32 * each
