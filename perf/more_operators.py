"""Timed cases of a K/V cache held in 4 bits, each one pass through public
entry points:

* ``append``: the fp32 QKV projection rotated, q rounded, K and V quantised
  into their cache entries (``lp.op_kv4_append``), and the same entries read
  back into an ordinary cache (``lp.op_kv4_read``);
* ``read``: whole contexts of the 4-bit cache back into an ordinary cache
  (``lp.op_kv4_read``);
* ``decode``: one token a row over the 4-bit cache
  (``lp.op_kv4_decode_attention``);
* ``prefill``: packed new tokens, causal, over the 4-bit cache
  (``lp.op_kv4_prefill_attention``).

With ``own`` false the same results come from elementary torch operations in
32 bits.  Model shapes are those of the package's configurations; lengths are
those of its workloads (prompts of 16 to 4,096 tokens, up to 64 running
requests) and the longer contexts that a smaller cache makes room for.

The cache: for each block of 64 positions and KV head 72 * head_dim bytes, K
codes [64][hd / 2], K scales [64][hd / 32] fp16, V codes [16][hd / 8][4][4]
(four positions' words side by side), V scales [hd / 32][64] fp16.  A code is
a sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6; 32 dims share a scale, and
magnitudes end at 6 * 10752.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 64  # positions of a cache block
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# query heads, key/value heads, head_dim
HEADS = {"tiny": (4, 4, 64), "7b": (32, 32, 128), "8b": (32, 8, 128), "13b": (40, 40, 128), "70b": (64, 8, 128)}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # a decode step's new K and V, one row a request: latency alone
        dict(name="append 64 rows", kind="append", model="8b", requests=64, new_mean=1, pad=0, dtype="f16"),
        # a packed prefill step of many prompts
        dict(name="append 9 prompts", kind="append", model="8b", requests=9, new_mean=469, pad=2, dtype="bf16"),
        # the fp32 model's short conversation brought back for exact attention
        dict(name="read 1 context fp32", kind="read", model="tiny", requests=1, ctx_mean=130, pad=0, dtype="f32"),
        # parked conversations that come back into the 16-bit cache together
        dict(name="read 16 contexts", kind="read", model="13b", requests=16, ctx_mean=1500, pad=3, dtype="bf16"),
        # one user alone: the smallest batch
        dict(name="decode 1 row", kind="decode", model="8b", rows=1, ctx_mean=613, pad=0, dtype="f16"),
        # the fp32 model's batch
        dict(name="decode 8 rows fp32", kind="decode", model="tiny", rows=8, ctx_mean=130, pad=1, dtype="f32"),
        # a full batch of mixed contexts
        dict(name="decode 64 rows", kind="decode", model="8b", rows=64, ctx_mean=2300, pad=0, dtype="f16"),
        # a full batch of long contexts on the largest shape, what the smaller cache is for
        dict(name="decode 64 rows long", kind="decode", model="70b", rows=64, ctx_mean=8000, pad=0, dtype="bf16"),
        # the fp32 model's prompts
        dict(name="prefill 5 fp32", kind="prefill", model="tiny", requests=5, new_mean=20, cached_mean=64, dtype="f32"),
        # short questions that go on from conversations of their own
        dict(name="prefill 16 short", kind="prefill", model="8b", requests=16, new_mean=40, cached_mean=1500,
             dtype="f16"),
        # one typical prompt, every head with its own K and V
        dict(name="prefill 547", kind="prefill", model="7b", requests=1, new_mean=547, cached_mean=0, dtype="f16"),
        # a step of long prompts that go on from a context
        dict(name="prefill 3 long", kind="prefill", model="70b", requests=3, new_mean=2100, cached_mean=2000,
             dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "read", "decode", "decode", "prefill", "prefill"])
    half = rng.choice(["f16", "bf16"])
    tiny = rng.random() < 0.2
    model, dtype = ("tiny", rng.choice(["f32", half])) if tiny else (rng.choice(["7b", "8b", "8b", "13b", "70b"]), half)
    if kind == "append":
        one = rng.random() < 0.5
        requests = _log_int(rng, 1, 64)
        return dict(kind=kind, model=model, requests=requests,
                    new_mean=1 if one else _log_int(rng, 2, max(3, 2800 // requests)),
                    pad=rng.choice([0, 0, rng.randint(1, 20)]), dtype=dtype)
    if kind == "read":
        requests = _log_int(rng, 1, 32)
        return dict(kind=kind, model=model, requests=requests, ctx_mean=_log_int(rng, 1, min(4000, 20000 // requests)),
                    pad=rng.choice([0, 0, rng.randint(1, 20)]), dtype=dtype)
    if kind == "decode":
        top = {"tiny": 2000, "8b": 7000, "70b": 7000, "7b": 1500, "13b": 1200}[model]
        return dict(kind=kind, model=model, rows=_log_int(rng, 1, 64), ctx_mean=_log_int(rng, 1, top),
                    pad=rng.choice([0, 0, rng.randint(1, 4)]), dtype=dtype)
    requests = _log_int(rng, 1, 32)
    return dict(kind=kind, model=model, requests=requests,
                new_mean=_log_int(rng, 1, 100 if tiny else min(2100, 4200 // requests)),
                cached_mean=rng.choice([0, _log_int(rng, 1, 300 if tiny else 2000)]), dtype=dtype)


# ------------------------------------------------------------------ 4 bits in elementary operations

def _sections(cache):
    """Views of a cache [n, Hkv, 72 hd]: K codes [n, Hkv, 64, hd / 2], K scales [n, Hkv, 64, hd / 32], V codes
    [n, Hkv, 16, hd / 8, 4, 4], V scales [n, Hkv, hd / 32, 64]."""
    n, hkv, size = cache.shape
    hd = size // 72
    half = cache.view(torch.float16)
    return (cache[..., :32 * hd].view(n, hkv, BLOCK, hd // 2),
            half[..., 16 * hd:18 * hd].view(n, hkv, BLOCK, hd // 32),
            cache[..., 36 * hd:68 * hd].view(n, hkv, 16, hd // 8, 4, 4),
            half[..., 34 * hd:].view(n, hkv, hd // 32, BLOCK))


def _quantise(x):
    """Codes [..., hd] (uint8, 0 to 15) and scales [..., hd / 32] (fp16) of fp32 values; the scale in 64 bits, as amax
    / 6 lies on its grid for many exact inputs."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    amax = g.abs().amax(-1, keepdim=True)
    t = amax.double() / torch.full((), 6.0, dtype=torch.float64, device=x.device)
    step = torch.ldexp(torch.ones_like(t), torch.frexp(t).exponent - 6).clamp(min=2.0 ** -23)
    s = (torch.ceil(t / step) * step).clamp(max=10752.0)
    s = torch.where(amax.isfinite(), s, torch.full_like(s, math.nan)).float()
    a, u = g.abs(), torch.where(s > 0, s, torch.ones_like(s))  # all of a group of scale 0 is 0
    # the borders between neighbours; products of 6 and 3 bits are exact
    code = ((a > 0.25 * u).byte() + (a >= 0.75 * u).byte() + (a > 1.25 * u).byte() + (a >= 1.75 * u).byte()
            + (a > 2.5 * u).byte() + (a >= 3.5 * u).byte() + (a > 5.0 * u).byte())
    code += torch.signbit(g).byte() * 8
    return code.reshape(x.shape), s[..., 0].half()


def _pack_k(code):
    """Codes [..., hd] as bytes [..., hd / 2] in the order of a K row."""
    c = code.reshape(*code.shape[:-1], -1, 4, 4, 2)  # 32-dim group, octet of it, pair, dim
    b = c[..., 0] | (c[..., 1] << 4)
    return b.transpose(-3, -2).reshape(*code.shape[:-1], -1)


def _pack_v(code):
    """Codes [..., hd] as bytes [..., hd / 8, 4] in the order of a V row."""
    c = code.reshape(*code.shape[:-1], -1, 16, 2)  # 32-dim group, pair, dim
    b = c[..., 0] | (c[..., 1] << 4)
    return b.transpose(-1, -2).reshape(*code.shape[:-1], -1, 4)


def _values(code, scale):
    """Codes [..., hd] and scales [..., hd / 32] as fp32 values."""
    lut = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=code.device)
    v = lut[code.int()].reshape(*code.shape[:-1], -1, 32)
    return (v * scale.float()[..., None]).reshape(code.shape)


def _nibbles(b):
    return torch.stack([b & 15, b >> 4], dim=-1)


def _k_values(codes, scales):
    """K rows' bytes [..., hd / 2] and scales [..., hd / 32] as values [..., hd]."""
    c = _nibbles(codes.reshape(*codes.shape[:-1], 4, -1, 4)).transpose(-4, -3)
    return _values(c.reshape(*codes.shape[:-1], -1), scales)


def _v_values(codes, scales):
    """V's bytes [..., hd / 8, 4] and scales [..., hd / 32] as values [..., hd]."""
    c = _nibbles(codes.flatten(-2).unflatten(-1, (16, -1))).transpose(-3, -2)
    return _values(c.reshape(*codes.shape[:-2], -1), scales)


def _context(cache, blocks):
    """K and V, fp32 [*, Hkv, 64 blocks, hd], of lists of blocks [*, n]."""
    kc, ks, vc, vs = _sections(cache)
    k = _k_values(kc[blocks], ks[blocks])
    v = _v_values(vc[blocks].transpose(-3, -2).flatten(-4, -3), vs[blocks].transpose(-1, -2))
    # [*, n, Hkv, 64, hd]
    return [x.transpose(-4, -3).flatten(-3, -2) for x in (k, v)]


# ------------------------------------------------------------------ prepare

def _lengths(case, n, mean, salt):
    """n lognormal lengths of at least 1 whose mean is at most `mean`, a function of the case alone; all `mean` if it
    is 0 or 1."""
    if mean <= 1 or n == 1:
        return [mean] * n
    rng = random.Random("%s %d %d" % (salt, n, mean))
    draws = [math.exp(rng.gauss(0.0, 0.45)) for _ in range(n)]
    scale = min(1.0, n / sum(draws)) * mean
    return [max(1, int(x * scale)) for x in draws]


def _layout(case):
    """Per sequence of the case: positions cached before the step, new positions."""
    kind = case["kind"]
    if kind == "decode":
        return [x - 1 for x in _lengths(case, case["rows"], case["ctx_mean"], "ctx")], [1] * case["rows"]
    n = case["requests"]
    if kind == "read":
        return _lengths(case, n, case["ctx_mean"], "ctx"), [0] * n
    new = _lengths(case, n, case["new_mean"], "new")
    if kind == "append":
        return [37 * i % 600 for i in range(n)], new
    return _lengths(case, n, case["cached_mean"], "before"), new


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + 1)
    return g


def _randn(shape, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEV).to(dtype)


def _i32(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


def _i64(a):
    return torch.tensor(np.asarray(a, dtype=np.int64), device=DEV)


def _table(lengths, seed):
    """Number of blocks of a cache, block table (slots in reverse order) of sequences of these lengths."""
    need = [-(-x // BLOCK) for x in lengths]
    n_blocks = sum(need) + 3
    perm = np.random.default_rng(seed).permutation(n_blocks).astype(np.int32)
    table, at = np.full((len(need), max(need) + 1), -1, dtype=np.int32), 0
    for j, k in enumerate(need):
        table[len(need) - 1 - j, :k] = perm[at:at + k]
        at += k
    return n_blocks, table


def _rows_of(table, spans, pad):
    """Positions and cache entries of the rows (first, count) of every sequence, -1 for `pad` more."""
    pos, entry = [], []
    for j, (c, x) in enumerate(spans):
        p = np.arange(c, c + x)
        pos.append(p)
        entry.append(table[len(spans) - 1 - j][p // BLOCK].astype(np.int64) * BLOCK + p % BLOCK)
    none = np.full(pad, -1)
    return np.concatenate(pos + [none]), np.concatenate(entry + [none])


def _random_cache(n_blocks, hkv, hd, gen):
    """A cache of quantised normal values; K's dims differ in size, as those of trained models do."""
    cache = torch.empty(n_blocks, hkv, 72 * hd, dtype=torch.uint8, device=DEV)
    size = torch.exp(0.5 * _randn((hkv, 1, hd), gen))
    size = size / size.square().mean(-1, keepdim=True).sqrt()
    per = max(1, (1 << 26) // (hkv * BLOCK * hd))
    for b in range(0, n_blocks, per):
        n = min(per, n_blocks - b)
        kc, ks, vc, vs = _sections(cache[b:b + n])
        code, scale = _quantise(_randn((n, hkv, BLOCK, hd), gen) * size)
        kc.copy_(_pack_k(code))
        ks.copy_(scale)
        code, scale = _quantise(_randn((n, hkv, BLOCK, hd), gen))
        vc.copy_(_pack_v(code).reshape(n, hkv, 16, 4, hd // 8, 4).transpose(3, 4))
        vs.copy_(scale.transpose(-1, -2))
    return cache


def _rope_tables(n_pos, hd):
    i = torch.arange(hd // 2, dtype=torch.float64, device=DEV)
    angle = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-2.0 * i / hd)
    return angle.cos().float(), angle.sin().float()


def _plain_cache(rows, hkv, hd, dtype):
    """An ordinary cache with room for `rows` positions."""
    n = -(-rows // BLOCK) + 1
    return (torch.zeros(n, hkv, BLOCK, hd, dtype=dtype, device=DEV),
            torch.zeros(n, hkv, hd, BLOCK, dtype=dtype, device=DEV))


def _prepare_append(case, seed):
    hq, hkv, hd = HEADS[case["model"]]
    cached, new = _layout(case)
    n_blocks, table = _table([c + x for c, x in zip(cached, new)], seed)
    pos, entry = _rows_of(table, list(zip(cached, new)), case["pad"])
    g, dt, rows = _gen(seed), DTYPES[case["dtype"]], len(pos)
    cos, sin = _rope_tables(max(c + x for c, x in zip(cached, new)), hd)
    k, v = _plain_cache(rows, hkv, hd, dt)
    return {"qkv": _randn((rows, (hq + 2 * hkv) * hd), g), "cos": cos, "sin": sin, "pos": _i32(pos),
            "entry": _i64(entry), "to": _i64(np.where(pos >= 0, np.arange(rows), -1)), "heads": (hq, hkv, hd),
            "q": torch.zeros(rows, hq, hd, dtype=dt, device=DEV),
            "cache": torch.zeros(n_blocks, hkv, 72 * hd, dtype=torch.uint8, device=DEV), "k": k, "v": v}


def _prepare_read(case, seed):
    _, hkv, hd = HEADS[case["model"]]
    ctx, _ = _layout(case)
    n_blocks, table = _table(ctx, seed)
    _, entry = _rows_of(table, [(0, c) for c in ctx], case["pad"])
    # each context's positions from a block's beginning on, as the ordinary cache holds them
    to, at = [], 0
    for c in ctx:
        to.append(at + np.arange(c))
        at += -(-c // BLOCK) * BLOCK
    k, v = _plain_cache(at, hkv, hd, DTYPES[case["dtype"]])
    return {"cache": _random_cache(n_blocks, hkv, hd, _gen(seed)), "entry": _i64(entry),
            "to": _i64(np.concatenate(to + [np.full(case["pad"], -1)])), "k": k, "v": v}


def _prepare_attention(case, seed):
    hq, hkv, hd = HEADS[case["model"]]
    cached, new = _layout(case)
    n, pad = len(new), case.get("pad", 0)
    n_blocks, table = _table([c + x for c, x in zip(cached, new)], seed)
    g = _gen(seed)
    q = _randn((sum(new) + pad, hq, hd), g, DTYPES[case["dtype"]])
    return {"q": q, "out": torch.empty_like(q), "cache": _random_cache(n_blocks, hkv, hd, g), "table": _i32(table),
            "hkv": hkv, "max_ctx": max(c + x for c, x in zip(cached, new)), "max_new": max(new),
            "start": _i32(np.concatenate([[0], np.cumsum(new)])),
            "slot": _i32(np.concatenate([np.arange(n)[::-1], np.full(pad, -1)])),
            "pos": _i32(np.concatenate([cached, np.full(pad, -1)]))}


def prepare(case, seed):
    st = {"append": _prepare_append, "read": _prepare_read}.get(case["kind"], _prepare_attention)(case, seed)
    st["kind"] = case["kind"]
    return st


# ------------------------------------------------------------------ the plain forms

def _plain_read(st):
    live = (st["to"] >= 0).nonzero()[:, 0]
    src, dst = st["entry"][live], st["to"][live]
    kc, ks, vc, vs = _sections(st["cache"])
    b, p = src // BLOCK, src % BLOCK
    dt = st["k"].dtype
    st["k"][dst // BLOCK, :, dst % BLOCK] = _k_values(kc[b, :, p], ks[b, :, p]).to(dt)
    st["v"][dst // BLOCK, :, :, dst % BLOCK] = _v_values(vc[b, :, p // 4, :, p % 4], vs[b, :, :, p]).to(dt)
    return [st["k"], st["v"]]


def _plain_append(st):
    hq, hkv, hd = st["heads"]
    x = st["qkv"].view(-1, hq + 2 * hkv, hd)
    live = (st["pos"] >= 0).nonzero()[:, 0]
    x, pos = x[live], st["pos"][live].long()
    cos, sin = st["cos"][pos][:, None, :], st["sin"][pos][:, None, :]
    a, b = x[:, :hq + hkv, :hd // 2], x[:, :hq + hkv, hd // 2:]
    # one product rounded to 32 bits, the other exact in 64: a value next to a
    # border between two codes falls to the side that a fused step leaves it on
    c64, a64, b64 = cos.double(), a.double(), b.double()
    r = torch.cat([(a64 * c64 - (b * sin).double()).float(), (b64 * c64 + (a * sin).double()).float()], dim=-1)
    st["q"][live] = r[:, :hq].to(st["q"].dtype)
    kc, ks, vc, vs = _sections(st["cache"])
    entry = st["entry"][live]
    blk, p = entry // BLOCK, entry % BLOCK
    code, scale = _quantise(r[:, hq:])
    kc[blk, :, p] = _pack_k(code)
    ks[blk, :, p] = scale
    code, scale = _quantise(x[:, hq + hkv:])
    vc[blk, :, p // 4, :, p % 4] = _pack_v(code)
    vs[blk, :, :, p] = scale
    return [st["q"]] + _plain_read(st)


def _softmax_of(q, k, v, seen):
    """softmax(q k^T / sqrt(hd)) v over `seen` keys; rows that see none give 0."""
    s = (q @ k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(q.shape[-1]))
    s = torch.where(seen, s, torch.full((), -math.inf, device=s.device))
    m = s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    e = torch.exp(s - m)
    total = e.sum(-1, keepdim=True)
    return (e @ v) / torch.where(total > 0, total, torch.ones((), device=s.device))


def _padded(st, slot, pos, q):
    """Attention of sequences' rows q [n, new, Hq, hd] at positions pos [n, new]."""
    hkv, (n, new, hq, hd) = st["hkv"], q.shape
    group = hq // hkv
    blocks = st["table"][slot.clamp(min=0)][:, :-(-st["max_ctx"] // BLOCK)].long().clamp(min=0)
    k, v = _context(st["cache"], blocks)
    qo = q.float().view(n, new, hkv, group, hd).permute(0, 2, 1, 3, 4).reshape(n, hkv, new * group, hd)
    seen = torch.arange(k.shape[2], device=q.device) <= pos.repeat_interleave(group, dim=1)[:, None, :, None]
    o = _softmax_of(qo, k, v, seen)
    return o.view(n, hkv, new, group, hd).permute(0, 2, 1, 3, 4).reshape(n, new, hq, hd)


def _plain_decode(st):
    pos, slot = st["pos"].long()[:, None], st["slot"].long()
    per = max(1, (1 << 31) // (st["hkv"] * st["q"].shape[2] * st["max_ctx"]))  # rows whose padded contexts fit
    for b in range(0, len(slot), per):
        st["out"][b:b + per] = _padded(st, slot[b:b + per], pos[b:b + per], st["q"][b:b + per, None])[:, 0].to(
            st["out"].dtype)
    return st["out"]


def _plain_prefill(st):
    start, first, slot = st["start"].long(), st["pos"].long(), st["slot"].long()
    rows = torch.arange(st["q"].shape[0], device=start.device)
    i = torch.arange(st["max_new"], device=start.device)[None, :]
    take = (start[:-1, None] + i).clamp(max=len(rows) - 1)
    o = _padded(st, slot, first[:, None] + i, st["q"][take])
    j = torch.searchsorted(start[1:].contiguous(), rows, right=True)
    st["out"].copy_(o[j, rows - start[j]].to(st["out"].dtype))
    return st["out"]


# ------------------------------------------------------------------ the framework's calls

def _own_append(lp, st):
    lp.op_kv4_append(st["qkv"], st["cos"], st["sin"], st["pos"], st["entry"], st["q"], st["cache"])
    return [st["q"]] + _own_read(lp, st)


def _own_read(lp, st):
    lp.op_kv4_read(st["cache"], st["entry"], st["to"], st["k"], st["v"])
    return [st["k"], st["v"]]


def _own_decode(lp, st):
    rows, hq, hd = st["q"].shape
    if "ws" not in st:  # a program allocates its workspace once
        need = lp.kv4_decode_attention_ws_bytes(rows, hq, st["hkv"], hd, st["max_ctx"])
        st["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    lp.op_kv4_decode_attention(st["q"], st["out"], st["cache"], st["table"], st["slot"], st["pos"], st["max_ctx"],
                               st["ws"])
    return st["out"]


def _own_prefill(lp, st):
    rows, hq, hd = st["q"].shape
    if "ws" not in st:
        need = lp.kv4_prefill_attention_ws_bytes(rows, hq, st["hkv"], hd, st["max_ctx"])
        st["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    lp.op_kv4_prefill_attention(st["q"], st["out"], st["cache"], st["table"], st["start"], st["slot"], st["pos"],
                                st["max_new"], st["max_ctx"], st["ws"])
    return st["out"]


def run(st):
    if own:
        from paper_2410_02425_amd import lp
        return {"append": _own_append, "read": _own_read, "decode": _own_decode,
                "prefill": _own_prefill}[st["kind"]](lp, st)
    return {"append": _plain_append, "read": _plain_read, "decode": _plain_decode,
            "prefill": _plain_prefill}[st["kind"]](st)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    hq, hkv, hd = HEADS[case["model"]]
    cached, new = _layout(case)
    rows, kind = sum(new), case["kind"]
    size = 4 if case["dtype"] == "f32" else 2
    held = 2 * hkv * hd * 9 // 16  # bytes of a position: 4 bits a value, 2 bytes for 32
    if kind == "read":
        return {"bytes": sum(cached) * (held + 2 * hkv * hd * size + 16), "flops": 2 * sum(cached) * hkv * hd}
    if kind == "append":
        return {"bytes": rows * ((hq + 2 * hkv) * hd * 4 + 4 * hd + 28 + hq * hd * size + held + 2 * hkv * hd * size),
                "flops": rows * hd * (3 * (hq + hkv) + 4 * hkv)}
    seen = sum(c * x + x * (x + 1) // 2 for c, x in zip(cached, new))  # keys of all rows
    return {"bytes": (sum(cached) + rows) * held + 2 * rows * hq * hd * size, "flops": 4 * seen * hq * hd}


# ------------------------------------------------------------------ the definitions in 64 bits

def _nearest(x):
    """The values that 4 bits hold of x [..., hd] (float64), a group of 32 at a time: its scale is the least number of
    6 significant bits (a multiple of 2^-23) that is not below a sixth of the largest magnitude."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top / 6.0).clamp(min=-200.0)) - 5
    grid = torch.exp2(e.clamp(min=-23.0))
    m = torch.floor(top / 6.0 / grid)
    s = (torch.where(6.0 * m * grid < top, m + 1.0, m) * grid).clamp(max=10752.0)
    best, err = torch.zeros_like(g), g.abs()
    # even codes first, so that an odd one has to be nearer
    for mag in (1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):
        d = (g.abs() - mag * s).abs()
        near = d < err
        best, err = torch.where(near, mag * s, best), torch.where(near, d, err)
    return torch.copysign(best, g).reshape(x.shape)


def _exact_append(case, seed):
    st = _prepare_append(case, seed)
    hq, hkv, hd = st["heads"]
    half = hd // 2
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    x = st["qkv"].double().view(-1, hq + 2 * hkv, hd)
    keep = [r for r, p in enumerate(st["pos"].tolist()) if p >= 0]
    pos = st["pos"].long()[keep]
    # the pair (i, i + hd/2) as a complex number, turned by its angle
    turn = torch.complex(st["cos"].double()[pos], st["sin"].double()[pos])[:, None, :]
    z = torch.complex(x[keep, :hq + hkv, :half], x[keep, :hq + hkv, half:]) * turn
    r = torch.cat([z.real, z.imag], dim=2)
    q[keep] = r[:, :hq]
    at = st["to"][keep]
    for h in range(hkv):
        k[:, h][at // BLOCK, at % BLOCK] = _nearest(r[:, hq + h])
        v[:, h][at // BLOCK, :, at % BLOCK] = _nearest(x[keep, hq + hkv + h])
    return [q, k, v]


def _exact_context(cache, blocks, h):
    """K and V [64 blocks, hd] of one head in 64 bits, byte by byte from the layout."""
    hd = cache.shape[2] // 72
    raw = cache[blocks.long(), h]
    n = raw.shape[0]
    mags = torch.tensor(MAGNITUDES, dtype=torch.float64, device=cache.device)

    def of(byte):
        return torch.stack([mags[(c & 7).long()] * (1 - 2 * (c >> 3).double()) for c in (byte & 15, byte >> 4)], -1)

    def scales(at):
        return raw[:, at:at + 4 * hd].contiguous().view(torch.float16).double()

    # K: octet i of group j of a row is at bytes hd / 8 i + 4 j
    k = of(raw[:, :32 * hd].reshape(n, BLOCK, 4, hd // 32, 4)).permute(0, 1, 3, 2, 4, 5).reshape(n, BLOCK, hd)
    k = k * scales(32 * hd).view(n, BLOCK, hd // 32).repeat_interleave(32, dim=2)
    # V: dims 32 j + 2 r and the next are at byte hd / 32 r + j of a row
    row = raw[:, 36 * hd:68 * hd].reshape(n, 16, hd // 8, 4, 4).permute(0, 1, 3, 2, 4).reshape(n, BLOCK, 16, hd // 32)
    v = of(row.transpose(2, 3)).reshape(n, BLOCK, hd)
    v = v * scales(68 * hd).view(n, hd // 32, BLOCK).transpose(1, 2).repeat_interleave(32, dim=2)
    return k.view(-1, hd), v.view(-1, hd)


def _exact_read(case, seed):
    st = _prepare_read(case, seed)
    k, v = st["k"].double(), st["v"].double()
    keep = st["to"] >= 0
    src, dst = st["entry"][keep], st["to"][keep]
    every = torch.arange(st["cache"].shape[0], device=DEV)
    for h in range(k.shape[1]):
        kk, vv = _exact_context(st["cache"], every, h)
        k[:, h][dst // BLOCK, dst % BLOCK] = kk[src]
        v[:, h][dst // BLOCK, :, dst % BLOCK] = vv[src]
    return [k, v]


def _exact_attention(case, seed):
    st = _prepare_attention(case, seed)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    group = out.shape[1] // st["hkv"]
    start = st["start"].tolist()
    for j, (s, p) in enumerate(zip(st["slot"].tolist(), st["pos"].tolist())):
        if p < 0:
            continue
        lo, hi = start[j], start[j + 1]
        top = p + hi - lo
        ahead = torch.arange(top, device=DEV)[None, :] > p + torch.arange(hi - lo, device=DEV)[:, None]
        for h in range(st["hkv"]):
            k, v = _exact_context(st["cache"], st["table"][s, :-(-top // BLOCK)], h)
            for i in range(h * group, (h + 1) * group):
                w = st["q"][lo:hi, i].double() @ k[:top].T / math.sqrt(k.shape[1])
                out[lo:hi, i] = torch.softmax(w.masked_fill(ahead, -math.inf), dim=1) @ v[:top]
    return out


def exact(case, seed):
    return {"append": _exact_append, "read": _exact_read}.get(case["kind"], _exact_attention)(case, seed)
