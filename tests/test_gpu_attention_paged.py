"""dg_attention_paged: against the CPU oracle's attention bit for bit where the
orders meet (one span, the library's exponential), against the softmax in 64
bits elsewhere, and against itself in other chunks, batches, pages, layouts and
launches, where a row's bits have to stay.

The bound against 64 bits, with A = sum p |v| / sum p: the probabilities are
rounded once, by at most u = half a step of their type; a score is a sum of d
products in chunks of 8, each cut at 2^-23 of the largest, so off by at most
d / 8 x 2^-23 S, S = max_t sum |q k_t| scaled, and its exponential by ln 2 of that,
above and below the division, with 2 x 2^-23 |s| <= 2^-22 S of the scaling and
subtraction; n keys join the output by n / 8 such chunks and the sum by n / 64
blocks, spans by two roundings each; then the output's own rounding.
"""
import itertools
import math

import numpy as np
import pytest

import oracle
from paper_2609_11356_amd import inputs
from tests.gpu_util import assert_bits_equal, dev_bf16, host_bits

pytestmark = pytest.mark.gpu

LOG2E = 1.4426950408889634


@pytest.fixture(scope="module")
def dg():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_11356_amd import dg as _dg
    _dg.lib()
    return _dg


def scale(d):
    return float(np.float32(LOG2E / math.sqrt(d)))


class Batch:
    """A ragged batch over a cache whose pages lie anywhere; cache places that no
    sequence has hold NaN."""

    def __init__(self, dg, q_lens, kv_lens, Hq=4, Hkv=2, dim=64, dtype="bfloat16", cache=None, page=16, seed=0,
                 behind=0, heads_first=False, k_scale=1.0, v_scale=1.0, dense=None):
        import torch
        self.q_lens, self.kv_lens, self.page, self.dim = q_lens, kv_lens, page, dim
        self.Hq, self.Hkv = Hq, Hkv
        dt = getattr(torch, dtype)
        ct = getattr(torch, cache) if cache else dt
        g = torch.Generator().manual_seed(seed)
        rows = sum(q_lens)
        if dense is None:
            dense = [torch.randn(n, 2, Hkv, dim, generator=g) for n in kv_lens]
            if ct.itemsize == 1:
                dense = [(d / torch.tensor([k_scale, v_scale]).view(1, 2, 1, 1)).clamp(-448, 448).to(ct).float() for d in dense]
            dense = [d.to(ct) for d in dense]
            self.q = (torch.randn(rows + behind, Hq, dim, generator=g) * 1.5).to(dt)
        else:
            dense, self.q = dense
        self.dense = dense
        need = [-(-n // page) for n in kv_lens]
        total = sum(need) + 2
        order = torch.randperm(total, generator=g)
        width = max(need + [1])
        table = torch.full((len(q_lens), width), -1, dtype=torch.int32)
        shape = (total, Hkv, page, dim) if heads_first else (total, page, Hkv, dim)
        store = []
        for _ in range(2):
            s = torch.full(shape, 0xff, dtype=torch.uint8) if ct.itemsize == 1 else torch.full(shape, float("nan"), dtype=ct)
            s = s.view(ct)
            store.append(s.transpose(1, 2) if heads_first else s)
        at = 0
        bytes_of = (lambda t: t.view(torch.uint8)) if ct.itemsize == 1 else (lambda t: t)
        for b, n in enumerate(kv_lens):
            for j in range(need[b]):
                p = int(order[at + j])
                table[b, j] = p
                part = dense[b][j * page:(j + 1) * page]
                for i in range(2):
                    bytes_of(store[i])[p, :len(part)] = bytes_of(part)[:, i]
            at += need[b]
        dev = [s.transpose(1, 2).contiguous().cuda().transpose(1, 2) if heads_first else s.cuda() for s in store]
        self.cache = dg.KvCache(dev[0], dev[1], k_scale, v_scale)
        self.k_scale, self.v_scale = k_scale, v_scale
        self.table = table.cuda()
        self.cu = torch.tensor([0] + list(np.cumsum(q_lens)), dtype=torch.int32).cuda()
        self.kv = torch.tensor(kv_lens, dtype=torch.int32).cuda()
        self.max_q, self.max_kv = max(q_lens + [0]), max(kv_lens + [0])

    def run(self, dg, desc, workspace=None, q=None, out=None, max_q=None, max_kv=None):
        import torch
        q = self.q.cuda() if q is None else q
        kind = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[desc.get("out", "bf16")]
        if out is None:
            out = torch.full(q.shape, 3.0, dtype=kind, device="cuda")
        return dg.dg_attention_paged(dg.AttnDesc(**desc), q, self.cache, self.cu, self.kv, self.table, out, scale(self.dim),
                                     self.max_q if max_q is None else max_q, self.max_kv if max_kv is None else max_kv,
                                     workspace=workspace)

    def space(self, dg, desc):
        import torch
        n = dg.dg_attention_paged_bytes(dg.AttnDesc(**desc), self.cache, self.q.shape[0], self.Hq, len(self.q_lens),
                                        self.max_q, self.max_kv)
        return torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")

    def exact(self, causal):
        """(answer, bound without the roundings of p and of the output, A) in 64 bits."""
        import torch
        rows, g = sum(self.q_lens), self.Hq // self.Hkv
        o = torch.zeros(rows, self.Hq, self.dim, dtype=torch.float64)
        A, rel = torch.zeros_like(o), torch.zeros(rows, self.Hq, 1, dtype=torch.float64)
        at = 0
        for b, (n, m) in enumerate(zip(self.q_lens, self.kv_lens)):
            if n and m:
                q = self.q[at:at + n].double()
                k = (self.dense[b][:, 0].double() * self.k_scale).repeat_interleave(g, 1)
                v = (self.dense[b][:, 1].double() * self.v_scale).repeat_interleave(g, 1)
                s = torch.stack([q[:, h] @ k[:, h].T for h in range(self.Hq)]) * (scale(self.dim) / LOG2E)
                S = torch.stack([q[:, h].abs() @ k[:, h].abs().T for h in range(self.Hq)]) * scale(self.dim)
                hide = torch.arange(m)[None] > m - n + torch.arange(n)[:, None] if causal else torch.zeros(n, m, dtype=torch.bool)
                p = torch.softmax(s.masked_fill(hide, -math.inf), -1).nan_to_num(0)
                S = S.masked_fill(hide, 0).amax(-1)
                o[at:at + n] = torch.stack([p[h] @ v[:, h] for h in range(self.Hq)], 1)
                A[at:at + n] = torch.stack([p[h] @ v[:, h].abs() for h in range(self.Hq)], 1)
                e = math.log(2) * 2 * S * (self.dim / 8 * 2.0 ** -23 + 2.0 ** -22) + (m / 8 + m / 64 + 32) * 2.0 ** -23
                rel[at:at + n, :, 0] = e.T
            at += n
        return o, rel, A


def check(batch, got, desc):
    import torch
    rows = sum(batch.q_lens)
    o, rel, A = batch.exact(desc.get("causal", 0))
    u_p = torch.finfo(torch.float16 if desc.get("p_dtype") == "f16" else torch.bfloat16).eps / 2
    kind = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[desc.get("out", "bf16")]
    u = torch.finfo(kind).eps / 2
    got = got[:rows].double().cpu()
    inner = A * (u_p + rel) * (1 + 2 * u_p)
    # binary16 probabilities below 2^-14 lose up to 2^-25 each, at |v| <= 6
    lost = 2.0 ** -25 * 6 * max(batch.kv_lens) if desc.get("p_dtype") == "f16" else 0.0
    bound = inner + u * (o.abs() + inner) + lost + torch.finfo(kind).smallest_normal * u
    bad = (got - o).abs() > bound
    assert not bad.any() and not got.isnan().any(), (int(bad.sum()), float(((got - o).abs() / bound.clamp(min=1e-30)).max()))


def same(a, b):
    import torch
    kind = torch.int16 if a.element_size() == 2 else torch.int32
    differ = int((a.view(kind) != b.view(kind)).sum())
    assert differ == 0, "%d of %d outputs differ" % (differ, a.numel())


# ------------------------------------------------------------ the oracle

ORDERS = [dict(causal=c, q_block=b, l_fma=lf, final=f, out=o)
          for (c, b), lf, (f, o) in itertools.product([(0, 64), (1, 64), (1, 128)], [0, 1], [("div", "bf16"), ("recip", "f32")])]


@pytest.mark.parametrize("oi", range(len(ORDERS)))
@pytest.mark.parametrize("H,L,dim", [(2, 1, 64), (1, 63, 128), (2, 130, 64), (1, 257, 128)])
def test_one_span_is_dg_attention(dg, oi, H, L, dim):
    """With the library's exponential and one span a whole prompt is dg_attention's
    answer, whose oracle it meets bit for bit."""
    import torch
    desc = dict(ORDERS[oi], key_block=64)
    Q, K, V = (inputs.normal_bf16(10 * oi + L + i, (H, L, dim), s) for i, s in enumerate((1.5, 1.5, 1.0)))
    want = oracle.attention(desc, Q, K, V, scale(dim))
    q = dev_bf16(Q).transpose(0, 1).contiguous().cpu()
    kv = torch.stack([dev_bf16(K).transpose(0, 1), dev_bf16(V).transpose(0, 1)], 1).contiguous().cpu()
    b = Batch(dg, [L], [L], Hq=H, Hkv=H, dim=dim, dense=([kv], q))
    assert_bits_equal(host_bits(b.run(dg, desc).transpose(0, 1).contiguous()), want, "%s %s" % (desc, (H, L, dim)))
    if L > 64:
        # the last tokens of the prompt as a chunk, and its last as a decoding step
        for n in (1, 40):
            part = Batch(dg, [n], [L], Hq=H, Hkv=H, dim=dim, dense=([kv], q[L - n:]))
            assert_bits_equal(host_bits(part.run(dg, desc).transpose(0, 1).contiguous()), want[:, L - n:], "last %d" % n)


# -------------------------------------------------------------- 64 bits

SHAPES = [  # new tokens, keys, query heads, key heads, head size
    ([1], [1], 1, 1, 64), ([1, 1, 1], [1001, 64, 65], 8, 2, 128), ([4, 1, 7], [300, 1, 7], 6, 2, 64),
    ([5], [700], 5, 1, 128), ([33, 2], [33, 515], 16, 1, 64), ([200, 1, 1], [450, 129, 128], 4, 2, 128),
    ([3, 0, 2, 5], [0, 40, 1, 2], 4, 4, 64), ([70], [1500], 8, 8, 128), ([130, 17], [130, 2000], 3, 3, 64),
]
TYPES = [("bfloat16", None, "bf16", "bf16"), ("float16", None, "f16", "f16"), ("bfloat16", "float8_e4m3fn", "bf16", "bf16"),
         ("bfloat16", None, "bf16", "f32")]


@pytest.mark.parametrize("exp2", ["inst", "lib"])
@pytest.mark.parametrize("ti", range(len(TYPES)))
@pytest.mark.parametrize("si", range(len(SHAPES)))
def test_against_64_bits(dg, si, ti, exp2):
    q, kv, Hq, Hkv, dim = SHAPES[si]
    dtype, cache, p, out = TYPES[ti]
    scales = (0.0625, 0.021) if cache else (1.0, 1.0)
    b = Batch(dg, q, kv, Hq, Hkv, dim, dtype, cache, page=(16, 7, 64, 1)[(si + ti) % 4], seed=si, behind=3,
              k_scale=scales[0], v_scale=scales[1])
    for causal, split in ((1, 0), (1, 128), (0, 256)):
        desc = dict(causal=causal, split_keys=split, exp2=exp2, p_dtype=p, out=out)
        got = b.run(dg, desc)
        check(b, got, desc)
        assert (got[sum(q):] == 3.0).all()          # rows behind the last sequence
        # rows that see nothing are zero
        at = 0
        for n, m in zip(q, kv):
            none = n if m == 0 else max(n - m, 0) if causal else 0
            assert (got[at:at + none] == 0).all()
            at += n
        # one workgroup for all of a row's spans: the same bits
        same(got, captured(b, dg, desc))
        # and a workspace of the caller's, whatever it held
        same(got, b.run(dg, desc, workspace=b.space(dg, desc)))


def captured(b, dg, desc, replays=1, workspace=None):
    """The same call from a graph (without a workspace: no records)."""
    import torch
    q = b.q.cuda()
    kind = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[desc.get("out", "bf16")]
    out = torch.full(q.shape, 3.0, dtype=kind, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            b.run(dg, desc, q=q, out=out, workspace=workspace)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(replays):
        out.fill_(3.0)
        graph.replay()
    torch.cuda.synchronize()
    return out


# -------------------------------------------------- the bits of a row

@pytest.mark.parametrize("exp2,split", [("inst", 256), ("lib", 128), ("inst", 0)])
@pytest.mark.parametrize("dtype,cache,p", [("bfloat16", None, "bf16"), ("float16", None, "f16"),
                                           ("bfloat16", "float8_e4m3fn", "bf16")])
def test_bits_do_not_depend_on_the_call(dg, exp2, split, dtype, cache, p):
    """One prompt of 700 tokens whole, in chunks and token by token, in other batches, pages
    and layouts, with bounds above its lengths: every row keeps its bits."""
    import torch
    n, Hq, Hkv, dim = 700, 8, 2, 128
    desc = dict(causal=1, split_keys=split, exp2=exp2, p_dtype=p, out=p)
    whole = Batch(dg, [n], [n], Hq, Hkv, dim, dtype, cache, seed=3)
    want = whole.run(dg, desc)
    dense, q = whole.dense[0], whole.q
    for first, size, page, heads_first in ((0, 1, 16, False), (64, 1, 5, True), (699, 1, 64, False), (512, 1, 128, False),
                                           (511, 1, 16, True), (300, 4, 48, False), (100, 16, 1, False), (250, 33, 16, True),
                                           (333, 200, 33, False), (0, 256, 64, False), (1, 699, 16, False)):
        end = first + size
        other = torch.randn(90, 2, Hkv, dim).to(dense.dtype)
        b = Batch(dg, [2, size, 1], [90, end, 77], Hq, Hkv, dim, dtype, cache, page=page, seed=first, heads_first=heads_first,
                  dense=([other, dense[:end], other[:77]], torch.cat([q[:2], q[first:end], q[:1]])))
        got = b.run(dg, desc, max_q=size + 500, max_kv=end + 3000)
        same(got[2:2 + size], want[first:end])
        same(b.run(dg, desc)[2:2 + size], want[first:end])
        alone = Batch(dg, [size], [end], Hq, Hkv, dim, dtype, cache, page=page, dense=([dense[:end]], q[first:end]))
        same(alone.run(dg, desc), want[first:end])


@pytest.mark.parametrize("dim,Hq,Hkv,n,m,cache", [(128, 64, 8, 820, 900, None), (128, 32, 8, 820, 900, None), (128, 64, 8, 810, 811, "float8_e4m3fn"),
                                                  (128, 16, 2, 130, 1300, None), (64, 64, 8, 820, 900, None), (64, 8, 1, 77, 2000, None)])
@pytest.mark.parametrize("exp2", ["inst", "lib"])
def test_bits_of_large_tiles(dg, dim, Hq, Hkv, n, m, cache, exp2):
    """Chunks whose tiles fill the chip, and some that nearly do, over several spans: every
    workgroup shape, against 64 bits, and the bits of single tokens and of one workgroup per row."""
    b = Batch(dg, [n], [m], Hq, Hkv, dim, "bfloat16", cache, seed=5)
    desc = dict(causal=1, split_keys=128, exp2=exp2)
    got = b.run(dg, desc)
    check(b, got, desc)
    same(got, captured(b, dg, desc))
    for j in (0, 1, 100 % n, n // 2, n - 1):
        part = Batch(dg, [1], [m - n + j + 1], Hq, Hkv, dim, "bfloat16", cache, dense=([b.dense[0][:m - n + j + 1]], b.q[j:j + 1]))
        same(part.run(dg, desc), got[j:j + 1])
    # the same chunk beside others: fewer and other tiles
    other = Batch(dg, [3, n, 1], [10, m, 5], Hq, Hkv, dim, "bfloat16", cache, seed=6,
                  dense=([b.dense[0][:10], b.dense[0], b.dense[0][:5]], torch_cat(b.q[:3], b.q, b.q[:1])))
    same(other.run(dg, desc)[3:3 + n], got)


def torch_cat(*parts):
    import torch
    return torch.cat(parts)


def test_decoding_by_appending(dg):
    """The operators together, as a program serves a prompt: a chunk is rotated and
    appended, attention reads the cache, then tokens follow one at a time from a
    captured step; every row has the bits of the prompt taken whole."""
    import torch
    n, first, Hq, Hkv, dim, page = 330, 300, 8, 2, 128, 16
    g = torch.Generator().manual_seed(9)
    qkv = torch.randn(n, Hq + 2 * Hkv, dim, generator=g).bfloat16().cuda()
    angle = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float64) / (dim // 2))
    cos, sin = angle.cos().float().cuda(), angle.sin().float().cuda()
    rope = dg.RopeDesc(dim)
    desc = dg.AttnDesc(causal=1, split_keys=128, exp2="inst")
    pages = 40
    table = torch.randperm(pages, generator=g)[:-(-n // page)].to(torch.int32)[None].cuda()

    def fresh():
        return dg.KvCache(*(torch.full((pages, page, Hkv, dim), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv"))

    def slots(a, b):
        t = torch.arange(a, b, device="cuda")
        return table[0, t // page].long() * page + t % page

    def serve(cache, x, pos, slot, cu, kv, most, max_kv, ws=None):
        q, k, v = x.split([Hq, Hkv, Hkv], 1)
        qr = torch.empty_like(q)
        dg.dg_kv_append(rope, k, v, pos, cos, sin, slot, cache, Q=q, Qout=qr)
        return dg.dg_attention_paged(desc, qr, cache, cu, kv, table, torch.zeros_like(qr), scale(dim), most, max_kv, workspace=ws)

    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")   # noqa: E731
    whole = serve(fresh(), qkv, torch.arange(n, dtype=torch.int32, device="cuda"), slots(0, n), i32(0, n), i32(n), n, n)
    cache = fresh()
    got = serve(cache, qkv[:first], torch.arange(first, dtype=torch.int32, device="cuda"), slots(0, first), i32(0, first),
                i32(first), first, first)
    same(got, whole[:first])
    x, pos, slot, cu, kv = qkv[:1].clone(), i32(0), slots(0, 1), i32(0, 1), i32(0)
    ws = torch.zeros(dg.dg_attention_paged_bytes(desc, cache, 1, Hq, 1, 1, n), dtype=torch.uint8, device="cuda")
    kv.fill_(0)
    slot.fill_(-1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        serve(cache, x, pos, slot, cu, kv, 1, n, ws)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            out = serve(cache, x, pos, slot, cu, kv, 1, n, ws)
        torch.cuda.synchronize()
    for t in range(first, n):
        x.copy_(qkv[t:t + 1])
        pos.fill_(t)
        kv.fill_(t + 1)
        slot.copy_(slots(t, t + 1))
        graph.replay()
        torch.cuda.synchronize()
        same(out, whole[t:t + 1])


# ------------------------------------------------------------- edges

def test_values_that_are_not_finite(dg):
    """Infinite and NaN keys and values reach the rows that see them and no other; a
    block whose scores are all -inf leaves the row to the others."""
    import torch
    n, m, H, dim = 4, 200, 2, 64
    for kind in ("inst", "lib"):
        for split in (0, 64):
            desc = dict(causal=1, split_keys=split, exp2=kind, out="f32")
            base = Batch(dg, [n], [m], H, H, dim, seed=1)
            clean = base.run(dg, desc)
            # the first block's keys score -inf against queries above zero
            q = base.q.abs() + 0.1
            dense = base.dense[0].clone()
            dense[:64, 0] = -math.inf
            b = Batch(dg, [n], [m], H, H, dim, dense=([dense], q))
            got = b.run(dg, desc)
            ref = Batch(dg, [n], [m - 64], H, H, dim, dense=([dense[64:]], q))
            same(got, ref.run(dg, desc))
            # every key -inf: 0 / 0
            dense[:, 0] = -math.inf
            assert Batch(dg, [n], [m], H, H, dim, dense=([dense], q)).run(dg, desc).isnan().all()
            # in a chunk of several tiles, at a value that some rows of one tile do not see
            long = Batch(dg, [150], [300], H, H, 128, seed=2)
            fine = long.run(dg, desc)
            dense = long.dense[0].clone()
            dense[210, 1, 1, 7], dense[290, 0, 0, 0] = math.nan, math.nan
            got = Batch(dg, [150], [300], H, H, 128, dense=([dense], long.q)).run(dg, desc)
            same(got[:60], fine[:60])
            same(got[:140, 0], fine[:140, 0])
            assert got[60:, 1, 7].isnan().all() and got[140:, 0].isnan().all()
            same(got[60:, 1, 8:], fine[60:, 1, 8:])
            # a NaN key, and an infinite value, that only the last row sees
            for i, bad in ((0, math.nan), (0, math.inf), (1, math.nan), (1, math.inf)):
                dense = base.dense[0].clone()
                dense[m - 1, i, 0, 5] = bad
                got = Batch(dg, [n], [m], H, H, dim, dense=([dense], base.q)).run(dg, desc)
                same(got[:n - 1], clean[:n - 1])
                same(got[:, 1], clean[:, 1])
                col = got[n - 1, 0, 5] if i else got[n - 1, 0]
                assert not col.isfinite().all() or (i == 0 and bad == math.inf and float(base.q[n - 1, 0, 5]) < 0)


def test_bad_pages_and_lengths(dg):
    """A page outside the cache is NaN to the rows that see its keys; lengths beyond the
    table, the bounds or the batch are cut."""
    import torch
    b = Batch(dg, [1, 3], [100, 60], 4, 2, 64, page=16, seed=2)
    for split in (0, 64):
        desc = dict(causal=1, split_keys=split, exp2="inst")
        want = b.run(dg, desc)
        good = b.table.clone()
        for bad in (-1, b.cache.pages, 1 << 30, -(1 << 31)):
            b.table.copy_(good)
            b.table[0, 5] = bad
            got = b.run(dg, desc)
            assert got[0].isnan().all()
            same(got[1:], want[1:])
        b.table.copy_(good)
        # keys past max_kv and past the table are not read
        b.kv[1] = 1 << 30
        got = b.run(dg, desc)
        same(got[:1], want[:1])
        b.kv[1] = -5
        got = b.run(dg, desc)
        assert (got[1:] == 0).all()
        b.kv[1] = 60
        # offsets that run backwards or past the rows
        b.cu[2] = 1 << 30
        same(b.run(dg, desc), want)
        b.cu[2] = 0
        got = b.run(dg, desc)
        same(got[:1], want[:1])
        assert (got[1:] == 3.0).all()
        b.cu[2] = 4


def test_bounds_below_the_lengths(dg):
    """New tokens past max_q are left as they are, keys past max_kv are not read."""
    import torch
    b = Batch(dg, [1, 3, 40], [300, 200, 260], 8, 2, 128, seed=12)
    for split in (0, 64):
        desc = dict(causal=1, split_keys=split, exp2="inst")
        want = b.run(dg, desc)
        got = b.run(dg, desc, max_q=2)
        same(got[:3], want[:3])
        same(got[4:6], want[4:6])
        assert (got[3:4] == 3.0).all() and (got[6:] == 3.0).all()
        got = b.run(dg, desc, max_kv=130)
        cut = b.kv.clamp(max=130)
        b.kv, keep = cut, b.kv
        same(got, b.run(dg, desc))
        b.kv = keep
        assert (b.run(dg, desc, max_kv=0) == 0).all()


def test_two_streams_and_two_threads_at_once(dg):
    """Calls of one descriptor and cache on two streams, each with a workspace of its own, and
    from two host threads on one stream."""
    import threading

    import torch
    desc = dict(causal=1, split_keys=64, exp2="inst")
    a = Batch(dg, [1] * 24, list(range(100, 2500, 100)), 8, 2, 128, seed=20)
    b = Batch(dg, [2, 30], [1900, 700], 8, 2, 128, seed=21)
    wanted = {x: x.run(dg, desc) for x in (a, b)}
    torch.cuda.synchronize()
    streams = {a: torch.cuda.Stream(), b: torch.cuda.Stream()}
    queries = {x: x.q.cuda() for x in (a, b)}
    torch.cuda.synchronize()
    got = {a: [], b: []}
    for _ in range(10):
        for x in (a, b):
            with torch.cuda.stream(streams[x]):
                got[x].append(x.run(dg, desc, q=queries[x]))
    torch.cuda.synchronize()
    for x in (a, b):
        for y in got[x]:
            same(y, wanted[x])
    one = torch.cuda.Stream()
    got = {a: [], b: []}

    def work(x):
        with torch.cuda.stream(one):
            for _ in range(10):
                got[x].append(x.run(dg, desc, q=queries[x]))

    threads = [threading.Thread(target=work, args=(x,)) for x in (a, b)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for x in (a, b):
        assert len(got[x]) == 10
        for y in got[x]:
            same(y, wanted[x])


def test_strides_and_streams(dg):
    """Queries inside a fused projection, outputs inside a wider row, a page table that is part
    of a wider one, on another stream than the current one."""
    import torch
    b = Batch(dg, [3, 40], [90, 300], 4, 2, 64, seed=4)
    desc = dict(causal=1, split_keys=128, exp2="inst")
    want = b.run(dg, desc)
    fused = torch.zeros(43, 9, 64, dtype=torch.bfloat16, device="cuda")
    fused[:, 2:6] = b.q.cuda()
    out = torch.full((4, 43, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    wide = torch.full((2, b.table.shape[1] + 5), 7, dtype=torch.int32, device="cuda")
    wide[:, 5:] = b.table
    b.table = wide[:, 5:]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run(dg, desc, q=fused[:, 2:6], out=out.transpose(0, 1)[..., :64])
    side.synchronize()
    same(out.transpose(0, 1)[..., :64].contiguous(), want)
    assert (out[..., 64:] == 3.0).all()


def test_offsets_past_32_bits(dg):
    """Sequences in the last pages of caches of over 2^32 bytes each."""
    import torch
    page, H, dim, n = 64, 8, 128, 500
    pages = (1 << 33) // (page * H * dim * 2) + 16
    small = Batch(dg, [2], [n], H, H, dim, seed=6, page=page)
    desc = dict(causal=1, split_keys=256, exp2="inst")
    want = small.run(dg, desc)
    K, V = (torch.zeros((pages, page, H, dim), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    for j in range(-(-n // page)):
        for big, part in ((K, small.cache.K), (V, small.cache.V)):
            big[pages - 1 - j] = part[int(small.table[0, j])]
        small.table[0, j] = pages - 1 - j
    small.cache = dg.KvCache(K, V)
    same(small.run(dg, desc), want)


def test_replays_with_other_lengths(dg):
    """A captured call reads its lengths when it runs: replayed on longer and shorter batches,
    with and without a workspace, and beside eager calls of the same stream."""
    import torch
    desc = dict(causal=1, split_keys=128, exp2="inst")
    b = Batch(dg, [1, 1, 1], [900, 500, 64], 8, 2, 128, seed=8)
    q = b.q.cuda()
    for ws in (None, b.space(dg, desc)):
        out = torch.zeros_like(q)
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                b.run(dg, desc, q=q, out=out, workspace=ws)
        torch.cuda.synchronize()
        for lens in ([900, 500, 64], [1, 2, 3], [129, 128, 0], [900, 1, 64]):
            b.kv.copy_(torch.tensor(lens, dtype=torch.int32))
            want = b.run(dg, desc)
            graph.replay()
            torch.cuda.synchronize()
            same(out, want)
        b.kv.copy_(torch.tensor([900, 500, 64], dtype=torch.int32))


def test_refusals(dg):
    import torch
    b = Batch(dg, [2], [20], 4, 2, 64)
    q = b.q.cuda()
    d = dg.AttnDesc(causal=1)
    ok = dict(desc=d, Q=q, cache=b.cache, cu_q=b.cu, kv_len=b.kv, page_table=b.table, O=torch.empty_like(q),
              qk_scale=0.1, max_q=2, max_kv=20)
    dg.dg_attention_paged(**ok)
    for bad in (dict(Q=q.half()), dict(Q=q[:, :3], O=q[:, :3].clone()), dict(O=q.float()), dict(O=q[:1]), dict(cu_q=b.cu.long()),
                dict(cu_q=b.cu[:1]), dict(kv_len=b.kv.cpu()), dict(page_table=b.table[0]), dict(page_table=b.table.long()),
                dict(Q=q.cpu()), dict(Q=q[..., :32], O=q[..., :32].clone()), dict(workspace=torch.zeros(64, device="cuda"))):
        with pytest.raises(ValueError):
            dg.dg_attention_paged(**dict(ok, **bad))
    for bad, status in ((dict(desc=dg.AttnDesc(key_block=32)), dg.DG_ERR_UNSUPPORTED), (dict(max_kv=-1), dg.DG_ERR_SHAPE),
                        (dict(O=q), dg.DG_ERR_INVALID), (dict(desc=dg.AttnDesc(exp2="inst"), qk_scale=0.0), dg.DG_ERR_INVALID)):
        with pytest.raises(dg.DgError) as e:
            dg.dg_attention_paged(**dict(ok, **bad))
        assert e.value.status == status
    long = dict(ok, desc=dg.AttnDesc(causal=1, split_keys=64), max_kv=128)
    with pytest.raises(dg.DgError) as e:
        dg.dg_attention_paged(**dict(long, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")))
    assert e.value.status == dg.DG_ERR_SCRATCH
