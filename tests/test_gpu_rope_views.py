"""dg_rope and dg_kv_append between views of one tensor that share no element: heads, halves
and tokens that lie between each other."""
import numpy as np
import pytest

from tests.test_gpu_rope import cuda, dg, host, rounded, same, tables, turn  # noqa: F401

pytestmark = pytest.mark.gpu


def views(t, dim):
    """(X, Y) inside t (tokens, 6, 2 dim) that share no element."""
    return {"heads that alternate": (t[:, ::2, :dim], t[:, 1::2, :dim]),
            "and the other way": (t[:, 1::2, :dim], t[:, ::2, :dim]),
            "heads behind each other": (t[:, :3, dim:], t[:, 3:, dim:]),
            "halves of a head": (t[..., :dim], t[..., dim:]),
            "tokens that alternate": (t[::2], t[1::2]),
            "the token before": (t[1:, :2], t[:-1, 4:]),
            "one head": (t[:, 2:3, :dim], t[:, 5:6, :dim]),
            "one token": (t[:1, ::2, :dim], t[:1, 1::2, dim:])}


@pytest.mark.parametrize("dim", [64, 36])
@pytest.mark.parametrize("name", list(views(np.zeros((4, 6, 2)), 1)))
def test_rotation_between_views(dg, name, dim):  # noqa: F811
    import torch
    t = torch.randn(10, 6, 2 * dim, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    x, y = views(t, dim)[name]
    d = x.shape[2]
    cos, sin = tables(20, d // 2, 2)
    pos = (np.arange(x.shape[0], dtype=np.int32) * 7 % 20)[None]
    want_x = host(x).copy()
    want = rounded(turn(want_x, pos, cos, sin, d, "half", None), x.dtype)
    rest = t.clone()
    views(rest, dim)[name][1].zero_()
    dg.dg_rope(dg.RopeDesc(d), x, cuda(pos), cuda(cos), cuda(sin), y)
    same(host(y), want)
    same(host(x), want_x)
    y.zero_()
    assert t.equal(rest)


def test_views_that_share_elements_are_refused(dg):  # noqa: F811
    import torch
    t = torch.zeros(10, 6, 128, dtype=torch.bfloat16, device="cuda")
    cos, sin = (cuda(a) for a in tables(20, 32))
    for x, y in ((t[:, :3, :64], t[:, 1:4, :64]), (t[:-1, ::2, :64], t[1:, ::2, :64]), (t[..., :64], t[..., 32:96]),
                 (t[:, ::2, :64], t[:, 1:4, :64]), (t[:5, :, :64], t[::2, :, 64:])):
        pos = torch.zeros(x.shape[0], dtype=torch.int32, device="cuda")
        with pytest.raises(dg.DgError) as e:
            dg.dg_rope(dg.RopeDesc(64), x, pos, cos, sin, y)
        assert e.value.status == dg.DG_ERR_INVALID


def test_queries_turn_beside_themselves(dg):  # noqa: F811
    """An append whose queries turn into heads of the same fused tensor."""
    import torch
    T, H, dim = 7, 3, 64
    t = torch.randn(T, 4 * H, dim, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    q, out, k, v = t.split(H, 1)
    cos, sin = tables(20, dim // 2, 5)
    pos = (np.arange(T, dtype=np.int32) * 3 % 20)[None]
    cache = dg.KvCache(*(torch.zeros(2, 4, H, dim, dtype=torch.bfloat16, device="cuda") for _ in "kv"))
    want = [rounded(turn(host(a), pos, cos, sin, dim, "half", None), t.dtype) for a in (q, k)]
    value = host(v).copy()
    dg.dg_kv_append(dg.RopeDesc(dim), k, v, cuda(pos), cuda(cos), cuda(sin), torch.arange(T, device="cuda"), cache, Q=q, Qout=out)
    same(host(out), want[0])
    same(host(cache.K).reshape(8, H, dim)[:T], want[1])
    same(host(cache.V).reshape(8, H, dim)[:T], value)
