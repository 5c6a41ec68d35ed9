"""dg_rope and dg_kv_append against the same steps in numpy's binary32, bit for
bit, and against the rotation in 64 bits.

y1 = RN(RN(x1 c) - RN(x2 s)) has three roundings to binary32 and one to its
type: |y - exact| <= u |exact| + 2^-24 (1 + u) 2.001 (|x1 c| + |x2 s|), u half a
step of the type relative to the value (bf16 2^-8, float16 2^-11, fp32 2^-24; plus
half of the type's smallest subnormal).  The gradient is the inverse rotation:
checked against the formula's transpose and against differences.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dg():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_11356_amd import dg as _dg
    _dg.lib()
    return _dg


def tables(rows, pairs, seed=0):
    """Angles of any kind: fp32 values, as they are data to the operator."""
    g = np.random.default_rng(seed)
    a = g.uniform(-math.pi, math.pi, (rows, pairs))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def turn(x, pos, cos, sin, rotary, pairing, axes, inverse=False, kind=np.float32):
    """x (T, H, dim) turned step by step in `kind`."""
    half = rotary // 2
    axes = np.zeros(half, int) if axes is None else np.asarray(axes)
    at = pos[axes].T                                              # (T, half)
    ok = (at >= 0) & (at < len(cos))
    col = np.arange(half)
    c = np.where(ok, cos[np.where(ok, at, 0), col], np.nan)[:, None].astype(kind)
    s = np.where(ok, sin[np.where(ok, at, 0), col], np.nan)[:, None].astype(kind)
    if inverse:
        s = -s
    y = x.astype(kind).copy()
    i0 = col if pairing == "half" else 2 * col
    i1 = col + half if pairing == "half" else 2 * col + 1
    a, b = x[..., i0].astype(kind), x[..., i1].astype(kind)
    y[..., i0] = a * c - b * s
    y[..., i1] = b * c + a * s
    return y


def host(t):
    return t.float().cpu().numpy()


def rounded(y, dtype):
    """binary32 values rounded once to a torch type, as binary32."""
    import torch
    return torch.from_numpy(y).to(dtype).float().numpy()


def same(got, want):
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.where(np.isnan(got), 0, got).view(np.uint32), np.where(np.isnan(want), 0, want).view(np.uint32))


CASES = [  # T, H, dim, rotary, pairing, axes kind, dtype
    (1, 1, 2, 2, "half", 1, "bfloat16"), (7, 3, 64, 64, "half", 1, "bfloat16"), (333, 5, 128, 128, "adjacent", 1, "float16"),
    (19, 9, 128, 64, "half", 3, "float32"), (65, 4, 64, 32, "adjacent", 2, "bfloat16"), (5, 33, 80, 80, "half", 3, "float16"),
    (4, 2, 96, 48, "half", 4, "bfloat16"), (3, 2, 36, 20, "adjacent", 2, "float32"), (130, 1, 512, 512, "half", 4, "bfloat16"),
    (11, 6, 72, 72, "half", "mixed", "bfloat16"), (9, 2, 128, 112, "adjacent", "mixed", "float16"), (1025, 32, 128, 128, "half", 3, "bfloat16"),
    # outputs past 32 MB
    (4200, 32, 128, 128, "half", 3, "bfloat16"), (2101, 32, 128, 96, "adjacent", 1, "float32"),
]


def make(case, seed):
    import torch
    T, H, dim, rotary, pairing, kind, dtype = case
    half = rotary // 2
    g = np.random.default_rng(seed)
    axes = (g.integers(0, 3, half).tolist() if kind == "mixed" else None if kind == 1 else
            [i * kind // half for i in range(half)])
    n = 1 if axes is None else max(axes) + 1
    cos, sin = tables(300, half, seed)
    pos = g.integers(0, 300, (n, T)).astype(np.int32)
    x = torch.from_numpy(g.standard_normal((T, H, dim)).astype(np.float32)).to(getattr(torch, dtype))
    return x, pos, cos, sin, axes


def cuda(a):
    import torch
    return torch.from_numpy(a).cuda()


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("ci", range(len(CASES)))
def test_rotation(dg, ci, inverse):
    import torch
    T, H, dim, rotary, pairing, _, dtype = CASES[ci]
    x, pos, cos, sin, axes = make(CASES[ci], ci)
    desc = dg.RopeDesc(dim, rotary, pairing, axes)
    xd, y = x.cuda(), torch.full_like(x, float("nan"), device="cuda")
    p, c, s = cuda(pos), cuda(cos), cuda(sin)
    dg.dg_rope(desc, xd, p, c, s, y, inverse=inverse)
    x32 = x.float().numpy()
    want = rounded(turn(x32, pos, cos, sin, rotary, pairing, axes, inverse), x.dtype)
    same(host(y), want)
    # in 64 bits
    exact = turn(x32.astype(np.float64), pos, cos, sin, rotary, pairing, axes, inverse, np.float64)
    size = np.abs(turn(np.abs(x32).astype(np.float64), pos, np.abs(cos), -np.abs(sin), rotary, pairing, axes, False, np.float64))
    size = np.maximum(size, np.abs(turn(np.abs(x32).astype(np.float64), pos, np.abs(cos), np.abs(sin), rotary, pairing, axes, False, np.float64)))
    u = torch.finfo(x.dtype).eps / 2
    tiny = torch.finfo(x.dtype).smallest_normal * u
    assert (np.abs(host(y) - exact) <= u * np.abs(exact) + 2.0 ** -24 * (1 + u) * 2.001 * size + tiny).all()
    # in place, and back at other strides: parts of wider rows, heads before tokens
    dg.dg_rope(desc, xd, p, c, s, xd, inverse=inverse)
    same(host(xd), want)
    wide = torch.full((T, H + 2, dim + 6), 7.0, dtype=x.dtype, device="cuda")
    wide[:, 1:H + 1, 3:dim + 3] = x.cuda()
    out = torch.full((H, T, dim + 8), 5.0, dtype=x.dtype, device="cuda")
    dg.dg_rope(desc, wide[:, 1:H + 1, 3:dim + 3], p, c, s, out.transpose(0, 1)[..., 8:], inverse=inverse)
    same(host(out.transpose(0, 1)[..., 8:]), want)
    assert (out[..., :8] == 5.0).all()


def test_gradient_by_formula_and_differences(dg):
    """<dY, rope(X)> as a function of X has the gradient rope^-1(dY); the map is
    linear, so a central difference of step 1 is exact up to its own rounding."""
    import torch
    case = (6, 2, 16, 12, "adjacent", 2, "float32")
    x, pos, cos, sin, axes = make(case, 3)
    desc = dg.RopeDesc(16, 12, "adjacent", axes)
    p, c, s = cuda(pos), cuda(cos), cuda(sin)
    dy = torch.randn(x.shape, generator=torch.Generator().manual_seed(1)).cuda()
    dx = dg.dg_rope(desc, dy, p, c, s, torch.empty_like(dy), inverse=True)
    f = lambda a: (dg.dg_rope(desc, a, p, c, s, torch.empty_like(a)).double() * dy.double()).sum()   # noqa: E731
    for i in range(0, x.numel(), 5):
        e = torch.zeros(x.numel(), device="cuda")
        e[i] = 1.0
        xd = x.cuda()
        diff = (f(xd + e.view_as(xd)) - f(xd - e.view_as(xd))) / 2
        # each of 2 x 384 terms is off by at most 3 x 2^-24 of values below 6 (x 6 of dy)
        assert abs(float(diff) - float(dx.flatten()[i])) < 4 * 2 * 2.0 ** -23 * 3 * 36


def test_positions_outside_the_tables_are_nan(dg):
    import torch
    desc = dg.RopeDesc(32, 16)
    cos, sin = tables(10, 8)
    x = torch.ones(4, 2, 32, dtype=torch.bfloat16, device="cuda")
    pos = torch.tensor([0, -1, 10, 9], dtype=torch.int32, device="cuda")
    y = host(dg.dg_rope(desc, x, pos, cuda(cos), cuda(sin), torch.empty_like(x)))
    assert np.isnan(y[1:3, :, :16]).all() and not np.isnan(y[[0, 3]]).any() and (y[1:3, :, 16:] == 1).all()


@pytest.mark.parametrize("cache_type,dtype", [("bfloat16", "bfloat16"), ("float16", "float16"), ("float8_e4m3fn", "bfloat16")])
@pytest.mark.parametrize("dim,rotary,pairing,kind", [(128, 128, "half", 1), (64, 32, "adjacent", 3), (80, 72, "half", 2),
                                                     (128, 0, "half", 1)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_append(dg, cache_type, dtype, dim, rotary, pairing, kind, heads_first):
    import torch
    T, Hq, Hkv, page, pages = 37, 6, 2, 12, 9
    x, pos, cos, sin, axes = make((T, Hq + 2 * Hkv, dim, rotary or 2, pairing, kind, dtype), 7)
    desc = dg.RopeDesc(dim, rotary, pairing, axes) if rotary else None
    ct = getattr(torch, cache_type)
    scales = (0.0371, 0.25) if cache_type == "float8_e4m3fn" else (1.0, 1.0)
    x = x * 9
    x[3, Hq] = float("nan")
    x[4, Hq + Hkv, 1] = float("inf")
    g = torch.Generator().manual_seed(5)
    slots = torch.randperm(pages * page, generator=g)[:T]
    slots[5], slots[20], slots[36] = -1, pages * page, -9

    def store():
        b = torch.full((pages, Hkv, page, dim) if heads_first else (pages, page, Hkv, dim), 0x3a,
                       dtype=torch.uint8).cuda() if ct.itemsize == 1 else torch.full(
            (pages, Hkv, page, dim) if heads_first else (pages, page, Hkv, dim), 0.75, dtype=ct).cuda()
        b = b.view(ct)
        return b.transpose(1, 2) if heads_first else b

    cache = dg.KvCache(store(), store(), *scales)
    qkv = x.cuda()
    q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
    qo = torch.full((T, Hq, dim), float("nan"), dtype=x.dtype, device="cuda")
    p, c, s = cuda(pos), cuda(cos), cuda(sin)
    more = dict(Q=q, Qout=qo) if rotary else {}
    dg.dg_kv_append(desc, k, v, p, c, s, slots.cuda(), cache, **more)
    x32 = x.float().numpy()
    turned = turn(x32, pos, cos, sin, rotary, pairing, axes) if rotary else x32
    if rotary:
        same(host(qo), rounded(turned[:, :Hq], x.dtype))
        dg.dg_kv_append(desc, k, v, p, c, s, slots.cuda(), cache, Q=q, Qout=q)       # in place
        same(host(q), rounded(turned[:, :Hq], x.dtype))
    for got, y, scale in ((cache.K, turned[:, Hq:Hq + Hkv], scales[0]), (cache.V, x32[:, Hq + Hkv:], scales[1])):
        want = store().cpu().float().numpy()
        if ct.itemsize == 1:
            z = np.clip(y / np.float32(scale), -448, 448).astype(np.float32)
            # torch's conversion rounds to nearest, ties to even
            z = rounded(z, ct)
        else:
            z = rounded(y, ct)
        for t in range(T):
            if 0 <= slots[t] < pages * page:
                want[slots[t] // page, slots[t] % page] = z[t]
        same(host(got), want)


def test_every_e4m3_rounding(dg):
    """All finite bf16 values through the 8-bit cache: round to nearest, ties to even, cut
    to +-448; infinities are cut, NaN stays."""
    import torch
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(512, 2, 64).cuda()
    K = torch.zeros((512, 1, 2, 64), dtype=torch.uint8, device="cuda")
    cache = dg.KvCache(K, torch.zeros_like(K))
    dg.dg_kv_append(None, bits, bits, None, None, None, torch.arange(512, device="cuda"), cache)
    x = bits.cpu().float()
    grid = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()      # 0 .. 448 upwards
    a = x.abs().double().clamp(max=448).flatten()
    i = torch.searchsorted(grid, a.nan_to_num(0)).clamp(max=126)
    lo, hi = grid[(i - 1).clamp(min=0)], grid[i]
    even_hi = i % 2 == 0
    up = (hi - a < a - lo) | ((hi - a == a - lo) & even_hi)
    want = torch.where(up, i, (i - 1).clamp(min=0))
    got = K.cpu().flatten()
    nan = x.flatten().isnan()
    assert ((got[nan] & 0x7f) == 0x7f).all()
    assert (got[~nan] & 0x7f).equal(want[~nan].to(torch.uint8))
    sign = torch.signbit(x.flatten())
    assert ((got[~nan] >> 7) == sign[~nan].to(torch.uint8)).all()
    assert cache.V.equal(K)


def test_offsets_past_32_bits(dg):
    """The last slot of caches of over 2^32 elements each."""
    import torch
    pages, page, H, dim = (1 << 32) // (64 * 8 * 128) + 3, 64, 8, 128
    K = torch.zeros((pages, page, H, dim), dtype=torch.uint8, device="cuda")
    cache = dg.KvCache(K, torch.zeros_like(K))
    k = torch.randn(2, H, dim, device="cuda").bfloat16()
    slots = torch.tensor([pages * page - 1, (1 << 32) // 1024 + 5], device="cuda")
    dg.dg_kv_append(None, k, k, None, None, None, slots, cache)
    want = k.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    for t in range(2):
        s = int(slots[t])
        assert K[s // page, s % page].equal(want[t]) and cache.V[s // page, s % page].equal(want[t])
    assert int((K[0] != 0).sum()) == 0 and int((K[pages // 2] != 0).sum()) == 0


def test_more_tokens_than_workgroups(dg):
    """2^20 workgroups take the tokens in turns."""
    import torch
    T, H, dim = (1 << 20) + 77, 3, 130
    cos, sin = tables(50, 65)
    x = torch.randn(T, H, dim, device="cuda").bfloat16()
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 50
    y = dg.dg_rope(dg.RopeDesc(dim), x, pos[None], cuda(cos), cuda(sin), torch.empty_like(x))
    for t in (0, 1, (1 << 20) - 1, 1 << 20, T - 1):
        want = turn(host(x[t:t + 1]), np.array([[t % 50]]), cos, sin, dim, "half", None)
        same(host(y[t:t + 1]), rounded(want, x.dtype))
    assert bool((y[1 << 20:] == dg.dg_rope(dg.RopeDesc(dim), x[1 << 20:], pos[None, 1 << 20:].contiguous(), cuda(cos), cuda(sin),
                                           torch.empty_like(x[1 << 20:]))).all())


def test_refusals(dg):
    import torch
    desc = dg.RopeDesc(64)
    cos, sin = (cuda(a) for a in tables(10, 32))
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    ok = dict(X=x, pos=pos, cos=cos, sin=sin, Y=torch.empty_like(x))
    dg.dg_rope(desc, **ok)
    for bad in (dict(X=x.double()), dict(X=x[..., :32]), dict(X=x.cpu()), dict(Y=x.float()), dict(Y=x[:3]), dict(X=x[0]),
                dict(pos=pos.long()), dict(pos=pos[:3]), dict(cos=cos.double()), dict(cos=cos[:, :16]), dict(sin=sin[:9]),
                dict(cos=cos.cpu()), dict(X=torch.zeros(4, 2, 128, dtype=x.dtype, device="cuda")[..., ::2])):
        with pytest.raises(ValueError):
            dg.dg_rope(desc, **dict(ok, **bad))
    with pytest.raises(dg.DgError):                       # rows of Y that share memory
        dg.dg_rope(desc, **dict(ok, Y=x[:1].expand(4, 2, 64)))
    with pytest.raises(dg.DgError):                       # half over X
        both = torch.zeros(5, 2, 64, dtype=x.dtype, device="cuda")
        dg.dg_rope(desc, **dict(ok, X=both[:4], Y=both[1:]))
    K = torch.zeros(3, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bad in ((K, K[:2]), (K, K.half()), (K.float(), K.float()), (K[..., ::2], K[..., ::2]), (K.cpu(), K.cpu()), (K[0], K[0])):
        with pytest.raises(ValueError):
            dg.KvCache(*bad)
    cache = dg.KvCache(K, K.clone())
    slots = torch.arange(4, device="cuda")
    ok = dict(desc=desc, K=x, V=x, pos=pos, cos=cos, sin=sin, slots=slots, cache=cache, Q=x, Qout=torch.empty_like(x))
    dg.dg_kv_append(**ok)
    for bad in (dict(K=x[:, :1]), dict(V=x.half()), dict(slots=slots.int()), dict(slots=slots[:3]), dict(Qout=None),
                dict(Q=x.half()), dict(desc=dg.RopeDesc(32)), dict(desc=None), dict(slots=slots.cpu())):
        with pytest.raises(ValueError):
            dg.dg_kv_append(**dict(ok, **bad))
    # empty calls
    dg.dg_rope(desc, x[:0], pos[:0], cos, sin, torch.empty_like(x[:0]))
    dg.dg_kv_append(desc, x[:0], x[:0], pos[:0], cos, sin, slots[:0], cache)
