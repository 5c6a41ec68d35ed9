"""Batches of dg_attention_paged whose spans and records are many: offsets that
start below the first row, contexts near the limit of keys, records taken in
turns, key heads that share an XCD, and values that are not finite in every
type and grouping.  Against 64 bits by the bound of test_gpu_attention_paged,
and against the same call in other launches, where the bits have to stay."""
import math

import pytest

from tests.test_gpu_attention_paged import LOG2E, Batch, captured, check, dg, same, scale  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,dim", [(4, 1, 64), (8, 2, 128)])
@pytest.mark.parametrize("split", [0, 64])
def test_offsets_below_the_first_row(dg, Hq, Hkv, dim, split):  # noqa: F811
    """An offset below 0 is brought to row 0 by the walk and by the join of its records."""
    b = Batch(dg, [20, 30], [200, 300], Hq, Hkv, dim, seed=31, behind=2)
    desc = dict(causal=1, split_keys=split, exp2="inst")
    want = b.run(dg, desc)
    check(b, want, desc)
    for first in (-1, -5, -(1 << 30), -(1 << 31)):
        b.cu[0] = first
        same(b.run(dg, desc), want)
        same(captured(b, dg, desc), want)
    # a sequence that ends below row 0 has no rows
    none = Batch(dg, [0, 20, 30], [200, 200, 300], Hq, Hkv, dim, seed=31,
                 dense=([b.dense[0]] + b.dense, b.q))
    clean = none.run(dg, desc)
    same(clean[:50], want[:50])
    none.cu[:2] = none.cu[:2] - 7
    none.cu[1] = -3
    same(none.run(dg, desc)[:50], clean[:50])


@pytest.mark.parametrize("Hq", [2, 20])
def test_as_many_keys_as_there_may_be(dg, Hq):  # noqa: F811
    """2^31 - 65536 keys: one page over and over, and at the end another that holds about half
    of the weight.  The bound is test_gpu_attention_paged's for the keys of one span, with two
    roundings of the sum and the output by every span on top."""
    import torch
    dim, page, split, n = 64, 8192, 131072, (1 << 31) - 65536
    g = torch.Generator().manual_seed(33)
    k = torch.randn(2, page, 1, dim, generator=g)
    k[1] = 1.55 + 0.05 * k[1]
    v = torch.randn(2, page, 1, dim, generator=g)
    v[1] += 1.0
    k, v = k.bfloat16(), v.bfloat16()
    q = (1.0 + 0.1 * torch.randn(1, Hq, dim, generator=g)).bfloat16()
    cache = dg.KvCache(k.cuda(), v.cuda())
    table = torch.zeros((1, n // page), dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")   # noqa: E731
    desc = dg.AttnDesc(causal=1, split_keys=split, exp2="inst", out="f32")
    got = dg.dg_attention_paged(desc, q.cuda(), cache, i32(0, 1), i32(n), table,
                                torch.full((1, Hq, dim), 3.0, device="cuda"), scale(dim), 1, n).double().cpu()[0]
    times = torch.tensor([n // page - 1, 1], dtype=torch.float64).repeat_interleave(page)
    kk, vv, qq = k.view(-1, dim).double(), v.view(-1, dim).double(), q[0].double()
    p = torch.softmax(qq @ kk.T * (scale(dim) / LOG2E) + times.log(), -1)
    assert 0.2 < float(p[:, page:].sum(1).min()) and float(p[:, page:].sum(1).max()) < 0.8
    S = (qq.abs() @ kk.abs().T).amax(1, keepdim=True) * scale(dim)
    rel = (math.log(2) * 2 * S * (dim / 8 * 2.0 ** -23 + 2.0 ** -22) + (split / 8 + split / 64 + 32) * 2.0 ** -23
           + n / split * 4 * 2.0 ** -24)
    bound = (p @ vv.abs()) * (2.0 ** -8 + rel) * (1 + 2.0 ** -7)
    assert not got.isnan().any()
    assert ((got - p @ vv).abs() <= bound).all(), float(((got - p @ vv).abs() / bound).max())


@pytest.mark.parametrize("Hq,Hkv", [(32, 1), (17, 1), (3, 1), (15, 3)])
def test_groups_that_16_rows_do_not_hold_whole(dg, Hq, Hkv):  # noqa: F811
    """Single tokens, drafted ones and a chunk of heads in groups of 32, 17, 3 and 5."""
    q = [1, 5, 1, 40, 3, 16]
    b = Batch(dg, q, [200, 333, 1, 500, 64, 129], Hq, Hkv, 64, seed=34)
    desc = dict(causal=1, split_keys=64, exp2="inst")
    want = b.run(dg, desc)
    check(b, want, desc)
    same(b.run(dg, desc, workspace=b.space(dg, desc)), want)
    same(captured(b, dg, desc), want)
    at = 0
    for i, n in enumerate(q):
        one = Batch(dg, [n], [b.kv_lens[i]], Hq, Hkv, 64, dense=([b.dense[i]], b.q[at:at + n]))
        same(one.run(dg, desc), want[at:at + n])
        at += n


@pytest.mark.parametrize("dim,Hq,Hkv,dtype,cache", [(64, 8, 8, "bfloat16", None), (64, 16, 8, "float16", None),
                                                    (128, 16, 8, "bfloat16", None), (128, 8, 8, "bfloat16", "float8_e4m3fn"),
                                                    (64, 12, 12, "bfloat16", "float8_e4m3fn")])
def test_neighbouring_heads_on_one_xcd(dg, dim, Hq, Hkv, dtype, cache):  # noqa: F811
    """Spans x sequences x key heads for some rounds of the chip: the heads of a span share an
    XCD and the spans' order turns from sequence to sequence."""
    lens = [1 + (149 * i) % 1100 for i in range(38)] + [1152]
    b = Batch(dg, [1 + i % 2 for i in range(39)], [n + 1 for n in lens], Hq, Hkv, dim, dtype, cache, page=32, seed=37,
              k_scale=0.0625 if cache else 1.0, v_scale=0.021 if cache else 1.0)
    p = "f16" if dtype == "float16" else "bf16"
    desc = dict(causal=1, split_keys=64, exp2="inst", p_dtype=p, out=p)
    assert -(-b.max_kv // 64) * 39 * Hkv >= 4096
    got = b.run(dg, desc)
    check(b, got, desc)
    same(got, captured(b, dg, desc))
    same(got, captured(b, dg, desc, replays=3, workspace=b.space(dg, desc)))


@pytest.mark.parametrize("exp2", ["inst", "lib"])
@pytest.mark.parametrize("kv", [[1024, 1025], [1088, 2112, 2560], [2049, 64, 65, 1]])
def test_more_spans_than_a_join_fetches_at_once(dg, kv, exp2):  # noqa: F811
    """16, 17, 33 and 40 spans, of few rows and of a chunk."""
    for q in ([1] * len(kv), [1] * (len(kv) - 2) + [24, 1]):
        b = Batch(dg, q, kv, 4, 2, 128, seed=39)
        desc = dict(causal=1, split_keys=64, exp2=exp2)
        got = b.run(dg, desc)
        check(b, got, desc)
        same(got, captured(b, dg, desc))


def test_two_streams_against_64_bits(dg):  # noqa: F811
    import torch
    desc = dict(causal=1, split_keys=64, exp2="inst")
    a = Batch(dg, [1] * 24, list(range(100, 2500, 100)), 8, 2, 128, seed=41)
    b = Batch(dg, [2, 30], [1900, 700], 8, 2, 128, seed=42)
    queries = {x: x.q.cuda() for x in (a, b)}
    streams = {a: torch.cuda.Stream(), b: torch.cuda.Stream()}
    torch.cuda.synchronize()
    got = {a: [], b: []}
    for _ in range(4):
        for x in (a, b):
            with torch.cuda.stream(streams[x]):
                got[x].append(x.run(dg, desc, q=queries[x]))
    torch.cuda.synchronize()
    for x in (a, b):
        check(x, got[x][0], desc)
        for y in got[x]:
            same(y, got[x][0])


@pytest.mark.parametrize("exp2,split", [("inst", 64), ("lib", 64), ("inst", 0)])
@pytest.mark.parametrize("g", [1, 3, 5])
@pytest.mark.parametrize("dtype,cache", [("bfloat16", None), ("float16", None), ("bfloat16", "float8_e4m3fn")])
def test_unseen_values_in_every_type(dg, dtype, cache, g, exp2, split):  # noqa: F811
    """NaN, infinite and the largest values reach the tokens that see them alone, in tiles whose
    rows are not whole tokens too, with records and with one workgroup for all of a row's spans."""
    import torch
    p = "f16" if dtype == "float16" else "bf16"
    desc = dict(causal=1, split_keys=split, exp2=exp2, p_dtype=p, out=p)
    for n, m, dim, at in ((3, 200, 64, 199), (4, 130, 128, 127), (150, 300, 128, 210), (70, 200, 64, 131)):
        base = Batch(dg, [n], [m], 2 * g, 2, dim, dtype, cache, seed=43 + n)
        clean = base.run(dg, desc)
        first = at - (m - n)                        # the first token that sees key `at`
        for bad in [math.nan, torch.finfo(base.dense[0].dtype).max] + ([] if cache else [math.inf]):
            dense = base.dense[0].clone()
            if cache:
                dense.view(torch.uint8)[at, 1, 0, 5] = 0x7f if math.isnan(bad) else 0x7e
            else:
                dense[at, 1, 0, 5] = bad
            b = Batch(dg, [n], [m], 2 * g, 2, dim, dtype, cache, dense=([dense], base.q))
            for got in (b.run(dg, desc), captured(b, dg, desc)):
                same(got[:first], clean[:first])
                same(got[:, g:], clean[:, g:])
                same(got[..., :5], clean[..., :5])
                same(got[..., 6:], clean[..., 6:])
                if math.isnan(bad):
                    assert got[first:, :g, 5].isnan().all()
                elif math.isinf(bad):
                    assert not got[first:, :g, 5].isfinite().any()


@pytest.mark.parametrize("exp2", ["inst", "lib"])
@pytest.mark.parametrize("split", [0, 128])
@pytest.mark.parametrize("q,kv", [([1700], [1800]), ([300, 1, 700, 850], [400, 1000, 900, 850])])
def test_large_chunks_over_e4m3(dg, q, kv, split, exp2):  # noqa: F811
    """Chunks that fill the chip in 256-row tiles, over a cache of 8 bits: against 64 bits, one
    workgroup for all of a row's spans, and single tokens."""
    b = Batch(dg, q, kv, 32, 8, 128, "bfloat16", "float8_e4m3fn", page=64, seed=45, k_scale=0.0625, v_scale=0.021, behind=1)
    desc = dict(causal=1, split_keys=split, exp2=exp2)
    got = b.run(dg, desc)
    check(b, got, desc)
    same(got, captured(b, dg, desc))
    at = 0
    for i, (n, m) in enumerate(zip(q, kv)):
        for j in (0, n // 2, n - 1):
            end = m - n + j + 1
            one = Batch(dg, [1], [end], 32, 8, 128, "bfloat16", "float8_e4m3fn", k_scale=0.0625, v_scale=0.021,
                        dense=([b.dense[i][:end]], b.q[at + j:at + j + 1]))
            same(one.run(dg, desc), got[at + j:at + j + 1])
        at += n
