"""The paged key/value cache and the rotation of positions: what is measured of them.

A case is one call that a program makes: rotating the queries or keys of a
training or encoder batch by positions with one to three axes (or the gradient
of that), appending new keys and values to a paged cache with the rotation on
the way, or attention of a ragged batch of new tokens over such a cache.  The
plain forms compute in 32 bits with elementary tensor operations and round
once; `exact` follows the definitions in 64 bits.

Head counts, head sizes and widths are those of the benchmark's layer (32 query
heads of 128 over 4096, 8 shared key heads) and generic ones around it.
"""
import functools
import math

import torch

own = False

LOG2E = 1.4426950408889634
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _rope(name=None, T=0, H=0, dim=128, rotary=None, pairing="half", axes=1, dtype="bf16", inverse=False):
    c = dict(op="rope", T=T, H=H, dim=dim, rotary=rotary or dim, pairing=pairing, axes=axes, dtype=dtype,
             inverse=inverse)
    return dict(c, name=name) if name else c


def _append(name=None, T=0, Hq=32, Hkv=8, dim=128, rotary=None, axes=1, dtype="bf16", cache="bf16", page=16, skip=0):
    c = dict(op="append", T=T, Hq=Hq, Hkv=Hkv, dim=dim, rotary=rotary or dim, axes=axes, dtype=dtype, cache=cache,
             page=page, skip=skip)
    return dict(c, name=name) if name else c


def _attn(name=None, B=1, q_min=1, q_max=1, kv_min=1, kv_max=1, Hq=32, Hkv=8, dim=128, dtype="bf16", cache=None,
          page=16, split=512, behind=0, long_one=0):
    """B sequences of q_min..q_max new tokens at the end of kv_min..kv_max cached keys (and where long_one is set
    one of them with that many new tokens), in a batch with `behind` rows after the last sequence."""
    c = dict(op="attention", B=B, q_min=q_min, q_max=q_max, kv_min=kv_min, kv_max=kv_max, Hq=Hq, Hkv=Hkv, dim=dim,
             dtype=dtype, cache=cache or dtype, page=page, split=split, behind=behind, long_one=long_one)
    return dict(c, name=name) if name else c


def listed():
    return [
        # queries of a training batch of text and video tokens: time, height and width
        _rope("rope_video_16384", T=16384, H=32, axes=3),
        # the gradient of an image encoder's rotation: two axes, adjacent pairs, an odd number of tokens
        _rope("rope_grad_image_4099", T=4099, H=16, dim=64, pairing="adjacent", axes=2, dtype="f16", inverse=True),
        # a short odd batch in 32 bits that rotates half of each head
        _rope("rope_partial_333", T=333, H=9, dim=128, rotary=64, dtype="f32"),
        # one decoding step of 64 sequences: rotate queries and keys, append
        _append("append_decode_64", T=64, skip=3),
        # a prompt's chunk into a cache of 8 bits, three axes
        _append("append_chunk_8192_e4m3", T=8192, axes=3, cache="e4m3", page=64),
        # one user, one token, a short context: the latency of a call, with short spans for it
        _attn("decode_1x1001", B=1, kv_min=1001, kv_max=1001, split=256),
        # a decoding batch with ragged contexts
        _attn("decode_64x4k", B=64, kv_min=200, kv_max=8000),
        # a larger one over a cache of 8 bits
        _attn("decode_128x8k_e4m3", B=128, kv_min=1000, kv_max=16000, cache="e4m3", page=64),
        # few sequences with long contexts
        _attn("decode_4x100k", B=4, kv_min=60000, kv_max=131072, page=32, split=1024),
        # checking four drafted tokens of 32 sequences, heads of 64
        _attn("verify_32x4", B=32, q_min=4, q_max=4, kv_min=300, kv_max=4500, Hq=16, Hkv=4, dim=64, dtype="f16"),
        # a chunk of a long prompt over what is cached of it
        _attn("chunk_4096_of_16k", B=1, q_min=4096, q_max=4096, kv_min=16000, kv_max=16000, page=32),
        # chunked prefill beside decoding sequences in one padded batch
        _attn("mixed_1023_and_11", B=12, kv_min=500, kv_max=8192, long_one=1023, behind=17),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention"])
    dim = rng.choice([64, 128, 128])
    if op == "rope":
        axes = rng.choice([1, 2, 3])
        H = rng.choice([1, 3, 8, 16, 32])
        return _rope(T=_log_int(rng, 1, 16384), H=H, dim=dim, rotary=rng.choice([dim, dim, dim // 2]),
                     pairing=rng.choice(["half", "adjacent"]), axes=axes, dtype=rng.choice(["bf16", "f16", "f32"])
                     if H < 32 else "bf16", inverse=rng.random() < 0.4)
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([n for n in (1, 2, 4, 5, 8, 16) if Hkv * n <= 32])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    cache = "e4m3" if dtype == "bf16" and rng.random() < 0.4 else dtype
    page = rng.choice([1, 16, 16, 48, 64, 128])
    if op == "append":
        return _append(T=_log_int(rng, 1, 8192), Hq=Hq, Hkv=Hkv, dim=dim, rotary=rng.choice([dim, dim, dim // 2]),
                       axes=rng.choice([1, 3]), dtype=dtype, cache=cache, page=page, skip=rng.choice([0, 2]))
    kind = rng.choice(["decode", "decode", "few", "chunk", "mixed"])
    split = rng.choice([256, 512, 1024])
    a = dict(Hq=Hq, Hkv=Hkv, dim=dim, dtype=dtype, cache=cache, page=page, split=split, behind=rng.choice([0, 0, 5]))
    if kind == "decode":
        B = _log_int(rng, 1, 128)
        kv = _log_int(rng, 1, min(131072, 128 * 8000 // B))
        return _attn(B=B, kv_min=max(1, kv // rng.choice([1, 2, 20])), kv_max=kv, **a)
    if kind == "few":
        kv = _log_int(rng, 40, 16000)
        q = rng.randint(2, 33)
        return _attn(B=_log_int(rng, 1, 32), q_min=rng.randint(1, q), q_max=q, kv_min=max(q, kv // 3), kv_max=max(q, kv), **a)
    if kind == "chunk":
        q = _log_int(rng, 64, 4096)
        kv = q + rng.choice([0, _log_int(rng, 1, 12000)])
        return _attn(B=1, q_min=q, q_max=q, kv_min=kv, kv_max=kv, **a)
    q = _log_int(rng, 64, 1024)
    kv = _log_int(rng, q, 8192)
    return _attn(B=rng.randint(2, 12), kv_min=max(1, kv // 4), kv_max=kv, long_one=q, **a)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(DTYPES[dtype])


def _pair_axes(pairs, axes):
    """The axis that turns each pair: runs for 3 axes in the ratio 1 : 1.5 : 1.5, equal ones otherwise."""
    if axes == 3:
        first = pairs // 4
        second = (pairs - first) // 2
        return [0] * first + [1] * second + [2] * (pairs - first - second)
    return [i * axes // pairs for i in range(pairs)]


def _tables(positions, pairs):
    f = 10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
    a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * f
    return a.cos().float(), a.sin().float()


def _positions(g, axes, T, table):
    """One axis: a run of positions far into the table; more: time, rows and columns of a grid of patches."""
    start = int(torch.randint(0, table - T + 1, (1,), generator=g, device="cuda"))
    t = torch.arange(T, device="cuda")
    if axes == 1:
        return (start + t).to(torch.int32)[None].contiguous()
    w, h = 23, 17
    grid = [t // (w * h), t // w % h, t % w]
    return torch.stack([start + x for x in grid[3 - axes:]]).to(torch.int32).contiguous()


def _spread(lo, hi, n):
    """n lengths evenly from lo to hi, the largest last."""
    return [hi - (n - 1 - i) * (hi - lo) // max(n - 1, 1) for i in range(n)]


def _lengths_of(case):
    """(new tokens, keys) of each sequence, before the seed puts them into an order."""
    B = case["B"]
    q, kv = _spread(case["q_min"], case["q_max"], B), _spread(case["kv_min"], case["kv_max"], B)
    if case["long_one"]:
        q[B // 2] = case["long_one"]
        kv[B // 2] = max(kv[B // 2], case["long_one"])
    return list(zip(q, kv))


def _lengths(case, g):
    pairs = _lengths_of(case)
    pairs = [pairs[i] for i in torch.randperm(len(pairs), generator=g, device="cuda").tolist()]
    return [q for q, _ in pairs], [kv for _, kv in pairs]


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["op"] in ("rope", "append"):
        T, pairs = case["T"], case["rotary"] // 2
        table = 32768
        s["cos"], s["sin"] = _tables(table, pairs)
        s["axes"] = _pair_axes(pairs, case["axes"])
        s["pair_axis"] = torch.tensor(s["axes"], device="cuda")
        s["pos"] = _positions(g, case["axes"], T, table)
    if case["op"] == "rope":
        s["x"] = _normal(g, (T, case["H"], case["dim"]), case["dtype"])
        s["y"] = torch.empty_like(s["x"])
        return s
    Hkv, dim, page = case["Hkv"], case["dim"], case["page"]
    kind = torch.float8_e4m3fn if case["cache"] == "e4m3" else DTYPES[case["cache"]]
    s["k_scale"], s["v_scale"] = (0.0625, 0.03125) if case["cache"] == "e4m3" else (1.0, 1.0)

    def cache_tensor(pages, scale):
        # filled in parts: a long cache's 32-bit draws are several times its size
        t = torch.empty((pages, page, Hkv, dim), dtype=kind, device="cuda")
        step = max(1, (1 << 26) // (page * Hkv * dim))
        for p in range(0, pages, step):
            part = t[p:p + step]
            part.copy_(torch.randn(part.shape, generator=g, device="cuda") / scale)
        return t

    if case["op"] == "append":
        # one fused projection's output: queries, keys and values side by side in each token's row
        qkv = _normal(g, (T, case["Hq"] + 2 * Hkv, dim), case["dtype"])
        s["q"], s["k"], s["v"] = qkv.split([case["Hq"], Hkv, Hkv], dim=1)
        s["q_out"] = torch.empty((T, case["Hq"], dim), dtype=qkv.dtype, device="cuda")
        pages = -(-4 * T // page) + 64
        s["k_cache"], s["v_cache"] = cache_tensor(pages, s["k_scale"]), cache_tensor(pages, s["v_scale"])
        # tokens lie in runs inside pages that are anywhere; the last ones of a padded batch go nowhere
        places = torch.randperm(pages, generator=g, device="cuda")[:, None] * page + torch.arange(page, device="cuda")
        s["slots"] = places.reshape(-1)[:T].contiguous()
        if case["skip"] and T > case["skip"]:
            s["slots"][T - case["skip"]:] = -1
        return s
    q, kv = _lengths(case, g)
    B, rows = case["B"], sum(q)
    s["max_q"], s["max_kv"] = max(q), max(kv)
    ends = torch.tensor([0] + q).cumsum(0)
    s["cu_q"] = ends.to(torch.int32).cuda()
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32).cuda()
    width = -(-s["max_kv"] // page)
    need = [-(-n // page) for n in kv]
    total = sum(need) + 3
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(width, device="cuda")[None] + torch.tensor([0] + need[:-1]).cumsum(0).cuda()[:, None]
    s["page_table"] = torch.where(torch.arange(width, device="cuda")[None] < torch.tensor(need).cuda()[:, None],
                                  order[at.clamp(max=total - 1)], torch.full((), -1, dtype=torch.int32, device="cuda"))
    s["page_table"] = s["page_table"].contiguous()
    s["k_cache"], s["v_cache"] = cache_tensor(total, s["k_scale"]), cache_tensor(total, s["v_scale"])
    s["q"] = _normal(g, (rows + case["behind"], case["Hq"], dim), case["dtype"], 1.5)
    s["o"] = torch.zeros_like(s["q"])
    return s


# ------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return {"rope": own_rope, "append": own_append, "attention": own_attention}[op](s)
    return {"rope": plain_rope, "append": plain_append, "attention": plain_attention}[op](s)


def _rotated(x, s, case, inverse=False):
    """x (T, H, dim) in the tables' type, each pair of it turned by its position's angle."""
    half = case["rotary"] // 2
    at = s["pos"][s["pair_axis"]].T.long()   # (T, pairs)
    col = torch.arange(half, device="cuda")
    c, sn = s["cos"][at, col][:, None].to(x.dtype), s["sin"][at, col][:, None].to(x.dtype)
    if inverse:
        sn = -sn
    if case.get("pairing", "half") == "half":
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * c - b * sn, b * c + a * sn, x[..., 2 * half:]], -1)
    a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    turned = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def plain_rope(s):
    case = s["case"]
    return _rotated(s["x"].float(), s, case, case["inverse"]).to(s["x"].dtype)


def _stored(x, cache, scale):
    if cache.dtype == torch.float8_e4m3fn:
        return (x / scale).clamp(-448.0, 448.0).to(cache.dtype)
    return x.to(cache.dtype)


def _appended(s, q, k, v):
    """Writes k and v at the slots (rows without one write the first row again) and returns the outputs."""
    case = s["case"]
    slots = s["slots"]
    row = torch.where(slots >= 0, torch.arange(case["T"], device="cuda"), torch.zeros_like(slots))
    page, place = slots[row] // case["page"], slots[row] % case["page"]
    for cache, x in ((s["k_cache"], k), (s["v_cache"], v)):
        # 8-bit elements are moved as bytes
        to = cache.view(torch.uint8) if cache.dtype == torch.float8_e4m3fn else cache
        to[page, place] = x.view(to.dtype)[row]
    return q, s["k_cache"], s["v_cache"]


def plain_append(s):
    case = s["case"]
    return _appended(s, _rotated(s["q"].float(), s, case).to(s["q"].dtype),
                     _stored(_rotated(s["k"].float(), s, case), s["k_cache"], s["k_scale"]),
                     _stored(s["v"].float(), s["v_cache"], s["v_scale"]))


def plain_attention(s):
    case = s["case"]
    B, Hq, Hkv, dim, page = (case[n] for n in ("B", "Hq", "Hkv", "dim", "page"))
    g = Hq // Hkv
    start, q_len, kv_len = s["cu_q"][:-1].long(), (s["cu_q"][1:] - s["cu_q"][:-1]).long(), s["kv_len"].long()
    t, j = torch.arange(s["max_kv"], device="cuda"), torch.arange(s["max_q"], device="cuda")
    # keys and values of each sequence side by side, short ones padded with zeros
    here = t < kv_len[:, None]
    pages = torch.where(here, s["page_table"][:, t // page].long(), 0)
    gather = lambda c: torch.where(here[..., None, None], c[pages, t % page].float(), 0.0).transpose(1, 2).contiguous()  # noqa: E731
    rows = (start[:, None] + j).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().view(B, -1, Hkv, g, dim).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, dim)
    scores = q @ (gather(s["k_cache"]).transpose(2, 3) * (s["k_scale"] / math.sqrt(dim)))
    last = kv_len[:, None] - q_len[:, None] + j                       # the last key that a query sees
    scores = scores.view(B, Hkv, -1, g, t.numel()).masked_fill_(
        (t > last[..., None])[:, None, :, None], -math.inf)
    scores = scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    scores = scores.div_(scores.sum(-1, keepdim=True)).view(B, Hkv, -1, t.numel())
    o = (scores @ gather(s["v_cache"])).mul_(s["v_scale"])
    o = o.view(B, Hkv, -1, g, dim).permute(0, 2, 1, 3, 4).reshape(B, -1, Hq, dim).to(s["q"].dtype)
    # back to the batch's rows; those behind the last sequence keep what they hold
    row = torch.arange(s["q"].shape[0], device="cuda")
    b = (torch.searchsorted(s["cu_q"].long(), row, right=True) - 1).clamp(max=B - 1)
    of = (row - start[b]).clamp(max=s["max_q"] - 1)
    return torch.where((row < s["cu_q"][-1])[:, None, None], o[b, of], s["o"])


@functools.lru_cache(maxsize=None)
def _dg():
    from paper_2609_11356_amd import dg
    return dg


@functools.lru_cache(maxsize=None)
def _rope_desc(dim, rotary, pairing, axes):
    return _dg().RopeDesc(dim=dim, rotary=rotary, pairing=pairing, axes=axes)


@functools.lru_cache(maxsize=None)
def _attn_desc(split, dtype):
    return _dg().AttnDesc(key_block=64, causal=1, q_block=64, split_keys=split, exp2="inst", p_dtype=dtype, out=dtype)


def _handle(s, make):
    """What a program keeps with its state between calls."""
    if "handle" not in s:
        s["handle"] = make()
    return s["handle"]


def _cache(s):
    return _dg().KvCache(s["k_cache"], s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def own_rope(s):
    c = s["case"]
    desc = _handle(s, lambda: _rope_desc(c["dim"], c["rotary"], c["pairing"], tuple(s["axes"])))
    return _dg().dg_rope(desc, s["x"], s["pos"], s["cos"], s["sin"], s["y"], inverse=c["inverse"])


def own_append(s):
    c = s["case"]
    desc, cache = _handle(s, lambda: (_rope_desc(c["dim"], c["rotary"], "half", tuple(s["axes"])), _cache(s)))
    _dg().dg_kv_append(desc, s["k"], s["v"], s["pos"], s["cos"], s["sin"], s["slots"], cache, Q=s["q"], Qout=s["q_out"])
    return s["q_out"], s["k_cache"], s["v_cache"]


def own_attention(s):
    c = s["case"]
    desc, cache = _handle(s, lambda: (_attn_desc(c["split"], c["dtype"]), _cache(s)))
    return _dg().dg_attention_paged(desc, s["q"], cache, s["cu_q"], s["kv_len"], s["page_table"], s["o"],
                                    LOG2E / math.sqrt(c["dim"]), max_q=s["max_q"], max_kv=s["max_kv"])


# ------------------------------------------------------- work and 64 bits

def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}
    dim = case["dim"]
    if case["op"] == "rope":
        n = case["T"] * case["H"] * dim
        return {"bytes": 2 * n * size[case["dtype"]] + case["T"] * case["rotary"] * 4, "flops": 3 * n}
    if case["op"] == "append":
        T, Hq, Hkv = case["T"], case["Hq"], case["Hkv"]
        moved = T * dim * (size[case["dtype"]] * (2 * Hq + 2 * Hkv) + size[case["cache"]] * 2 * Hkv)
        return {"bytes": moved + T * case["rotary"] * 4 + 8 * T, "flops": 3 * T * (Hq + Hkv) * dim}
    pairs = keys = new = 0
    for q, kv in _lengths_of(case):
        pairs += q * (kv - (q - 1) / 2)
        keys += kv
        new += q
    return {"bytes": 2 * keys * case["Hkv"] * dim * size[case["cache"]] + 2 * new * case["Hq"] * dim * size[case["dtype"]],
            "flops": 4 * pairs * case["Hq"] * dim}


def _turned_exactly(x, s, case, inverse):
    x = x.double().clone()
    of = torch.tensor(s["axes"]).tolist()
    for i, axis in enumerate(of):
        p = s["pos"][axis].long()
        c, sn = s["cos"][p, i].double()[:, None], s["sin"][p, i].double()[:, None]
        sn = -sn if inverse else sn
        u, v = (i, i + len(of)) if case.get("pairing", "half") == "half" else (2 * i, 2 * i + 1)
        a, b = x[..., u].clone(), x[..., v].clone()
        x[..., u], x[..., v] = a * c - b * sn, b * c + a * sn
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _turned_exactly(s["x"], s, case, case["inverse"])
    if case["op"] == "append":
        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        k, v = _turned_exactly(s["k"], s, case, False) / s["k_scale"], s["v"].double() / s["v_scale"]
        on = s["slots"] >= 0
        page, place = s["slots"][on] // case["page"], s["slots"][on] % case["page"]
        k_cache[page, place], v_cache[page, place] = k[on], v[on]
        return _turned_exactly(s["q"], s, case, False), k_cache, v_cache
    if work(case)["flops"] > 4e12:
        return None
    o = s["o"].double()
    g = case["Hq"] // case["Hkv"]
    ends, lengths = s["cu_q"].tolist(), s["kv_len"].tolist()
    for b, n in enumerate(lengths):
        t = torch.arange(n, device="cuda")
        page, place = s["page_table"][b, t // case["page"]].long(), t % case["page"]
        for h in range(case["Hkv"]):
            k = s["k_cache"][page, place, h].double() * s["k_scale"]
            v = s["v_cache"][page, place, h].double() * s["v_scale"]
            for at in range(ends[b], ends[b + 1], 1024):
                to = min(at + 1024, ends[b + 1])
                q = s["q"][at:to, h * g:(h + 1) * g].double().reshape(-1, case["dim"])
                last = n - ends[b + 1] + torch.arange(at, to, device="cuda").repeat_interleave(g)
                w = (q @ k.T.contiguous() / math.sqrt(case["dim"])).masked_fill(t > last[:, None], -math.inf)
                o[at:to, h * g:(h + 1) * g] = (torch.softmax(w, -1) @ v).view(to - at, g, -1)
    return o
