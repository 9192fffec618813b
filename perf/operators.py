"""Timed cases of serving a batch whose requests share a prefix, each one call
of a public entry point:

* ``tables``: a step's block tables, packed row offsets and cache entries from
  the requests' lengths (``lp.op_block_tables``);
* ``append``: the fp32 QKV projection rotated, q rounded, K and V stored at
  their cache entries (``lp.op_qkv_append``);
* ``decode``: one token a row over the shared prefix and the row's own context
  (``lp.op_prefix_decode_attention``);
* ``prefill``: packed new tokens over the shared prefix and their sequences'
  own context (``lp.op_prefix_prefill_attention``).

With ``own`` false the same results come from elementary torch operations in
32 bits.  Model shapes are those of the package's configurations; lengths are
those of its workloads (prompts of 16 to 4,096 tokens, up to 64 running
requests), and prefixes from a short instruction to a long document.
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


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # the tables of a full decode batch: one token a request, and a new
        # block for the few that fill theirs; latency alone
        dict(name="tables decode 64", kind="tables", requests=64, prefix=1024, ctx_mean=600, new_mean=1, pad=0),
        # admission of many requests at once, a step of about 65,000 tokens
        dict(name="tables admit 256", kind="tables", requests=256, prefix=2000, ctx_mean=0, new_mean=256, pad=500),
        # a full decode batch's new K and V, scattered over 64 blocks
        dict(name="append 64 rows", kind="append", model="8b", requests=64, new_mean=1, pad=0, dtype="f16"),
        # a packed prefill step of many prompts, in the other 16-bit type
        dict(name="append 9 prompts", kind="append", model="8b", requests=9, new_mean=469, pad=2, dtype="bf16"),
        # one user alone behind a service's instruction: the smallest batch
        dict(name="decode 1 row", kind="decode", model="8b", rows=1, prefix=553, own_mean=60, pad=0, dtype="f16"),
        # the fp32 model's batch over a short instruction
        dict(name="decode 8 rows fp32", kind="decode", model="tiny", rows=8, prefix=100, own_mean=30, pad=0,
             dtype="f32"),
        # a full batch over a system prompt of a few pages, own contexts mixed
        dict(name="decode 64 rows", kind="decode", model="8b", rows=64, prefix=2000, own_mean=300, pad=0, dtype="f16"),
        # many questions about one long document on the largest shape
        dict(name="decode 64 rows document", kind="decode", model="70b", rows=64, prefix=16000, own_mean=150, pad=0,
             dtype="bf16"),
        # the fp32 model's prompts behind its instruction
        dict(name="prefill 5 fp32", kind="prefill", model="tiny", requests=5, prefix=64, new_mean=20, cached_mean=0,
             dtype="f32"),
        # short questions that arrive together behind a system prompt
        dict(name="prefill 16 short", kind="prefill", model="8b", requests=16, prefix=1500, new_mean=40,
             cached_mean=0, dtype="f16"),
        # one typical prompt behind a document, every head with its own K and V
        dict(name="prefill 547 document", kind="prefill", model="7b", requests=1, prefix=4000, new_mean=547,
             cached_mean=0, dtype="f16"),
        # a step of long prompts that go on from a context of their own
        dict(name="prefill 3 long", kind="prefill", model="70b", requests=3, prefix=4096, new_mean=2100,
             cached_mean=300, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "append", "decode", "decode", "prefill", "prefill"])
    half = rng.choice(["f16", "f16", "bf16"])
    if kind == "tables":
        return dict(kind=kind, requests=_log_int(rng, 1, 256), prefix=_log_int(rng, 16, 8000),
                    ctx_mean=rng.choice([0, _log_int(rng, 16, 2000)]), new_mean=rng.choice([1, _log_int(rng, 2, 250)]),
                    pad=rng.choice([0, 0, rng.randint(1, 300)]))
    tiny = rng.random() < 0.2
    model, dtype = ("tiny", rng.choice(["f32", half])) if tiny else (rng.choice(["7b", "8b", "8b", "13b", "70b"]), half)
    if kind == "append":
        one = rng.random() < 0.5
        requests = _log_int(rng, 1, 64)
        return dict(kind=kind, model=model, requests=requests,
                    new_mean=1 if one else _log_int(rng, 2, max(3, 2800 // requests)),
                    pad=rng.choice([0, 0, rng.randint(1, 20)]), dtype=dtype)
    if kind == "decode":
        return dict(kind=kind, model=model, rows=_log_int(rng, 1, 64),
                    prefix=_log_int(rng, 16, 2000 if tiny else 16000), own_mean=_log_int(rng, 1, 300 if tiny else 600),
                    pad=rng.choice([0, 0, rng.randint(1, 4)]), dtype=dtype)
    requests = _log_int(rng, 1, 32)
    return dict(kind=kind, model=model, requests=requests, prefix=_log_int(rng, 16, 1000 if tiny else 4000),
                new_mean=_log_int(rng, 1, 100 if tiny else min(2100, 4200 // requests)),
                cached_mean=rng.choice([0, 0, _log_int(rng, 1, 400)]), dtype=dtype)


# ------------------------------------------------------------------ prepare

def _lengths(case, n, mean, salt):
    """n lognormal lengths of at least 1 whose mean is at most `mean`, a function of the case alone; all `mean` if it
    is 0 or 1."""
    if mean <= 1 or n == 1:
        return [mean] * n
    rng = random.Random("%s %d %d %d" % (salt, n, mean, case.get("prefix", 0)))
    draws = [math.exp(rng.gauss(0.0, 0.45)) for _ in range(n)]
    scale = min(1.0, n / sum(draws)) * mean
    return [max(1, int(x * scale)) for x in draws]


def _layout(case):
    """Per sequence of the case: positions cached before the step, new positions."""
    kind, prefix = case["kind"], case.get("prefix", 0)
    if kind == "decode":
        n = case["rows"]
        return [prefix + x - 1 for x in _lengths(case, n, case["own_mean"], "own")], [1] * n
    n = case["requests"]
    new = _lengths(case, n, case["new_mean"], "new")
    if kind == "append":
        return [37 * i % 600 for i in range(n)], new
    before = _lengths(case, n, case["ctx_mean" if kind == "tables" else "cached_mean"], "before")
    return [prefix + x for x in before], new


def _gen(seed, salt=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + salt)
    return g


def _randn(shape, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEV).to(dtype)


def _i32(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


def _tables_host(cached, new, prefix, perm):
    """Prefix blocks and block table (slots in reverse order) of sequences that
    hold their cached and new positions, out of the pool's blocks `perm`."""
    n_pre, first = -(-prefix // BLOCK), prefix // BLOCK
    need = [-(-(c + x) // BLOCK) for c, x in zip(cached, new)]
    wide = max(need + [n_pre]) + 1
    table = np.full((len(cached), wide), -1, dtype=np.int32)
    pre, at = perm[:n_pre], n_pre
    for j, k in enumerate(need):
        row = table[len(cached) - 1 - j]
        row[:min(first, k)] = pre[:min(first, k)]
        own_blocks = max(0, k - first)
        row[first:first + own_blocks] = perm[at:at + own_blocks]
        at += own_blocks
    return pre, table


def _blocks_needed(cached, new, prefix):
    return -(-prefix // BLOCK) + sum(-(-(c + x) // BLOCK) - prefix // BLOCK for c, x in zip(cached, new))


def _prepare_tables(case, seed):
    cached, new = _layout(case)
    n, prefix = len(cached), case["prefix"]
    first = prefix // BLOCK
    total = _blocks_needed(cached, new, prefix)
    perm = np.random.default_rng(seed).permutation(2 * total + 8).astype(np.int32)
    # what a program has before the step: tables that hold the cached positions
    pre, table = _tables_host(cached, [0] * n, prefix, perm)
    wide = max(-(-(c + x) // BLOCK) for c, x in zip(cached, new)) + 2
    full = np.full((n, wide), -1, dtype=np.int32)
    keep = min(wide, table.shape[1])
    full[:, :keep] = table[:, :keep]
    held = set(table[table >= 0].tolist()) | set(pre.tolist())
    free = np.array([b for b in perm.tolist() if b not in held], dtype=np.int32)
    for s in range(n):  # a new request's row is still empty
        if cached[n - 1 - s] <= prefix:
            full[s, :] = -1
    rows = sum(new) + case["pad"]
    return {"cached": _i32(cached), "lengths": _i32([c + x for c, x in zip(cached, new)]), "prefix_blocks": _i32(pre),
            "prefix_len": prefix, "free": _i32(free), "head": _i32([3]), "table": _i32(full),
            "slot": _i32(np.arange(n)[::-1].copy()), "first": first,
            "seq_start": torch.empty(n + 1, dtype=torch.int32, device=DEV),
            "free_start": torch.empty(n + 1, dtype=torch.int32, device=DEV),
            "row_slot": torch.empty(rows, dtype=torch.int32, device=DEV),
            "row_pos": torch.empty(rows, dtype=torch.int32, device=DEV),
            "row_entry": torch.empty(rows, dtype=torch.int64, device=DEV)}


def _rope_tables(n_pos, hd):
    i = torch.arange(hd // 2, dtype=torch.float64, device=DEV)
    angle = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-2.0 * i / hd)
    return angle.cos().float(), angle.sin().float()


def _prepare_append(case, seed):
    hq, hkv, hd = HEADS[case["model"]]
    cached, new = _layout(case)
    n_blocks = _blocks_needed(cached, new, 0) + 3
    perm = np.random.default_rng(seed).permutation(n_blocks).astype(np.int32)
    _, table = _tables_host(cached, new, 0, perm)
    pos, entry = [], []
    for j, (c, x) in enumerate(zip(cached, new)):
        p = np.arange(c, c + x)
        pos.append(p)
        entry.append(table[len(cached) - 1 - j][p // BLOCK].astype(np.int64) * BLOCK + p % BLOCK)
    pos.append(np.full(case["pad"], -1))
    entry.append(np.full(case["pad"], -1))
    pos, entry = np.concatenate(pos), np.concatenate(entry)
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    cos, sin = _rope_tables(max(c + x for c, x in zip(cached, new)), hd)
    rows = len(pos)
    return {"qkv": _randn((rows, (hq + 2 * hkv) * hd), g), "cos": cos, "sin": sin, "pos": _i32(pos),
            "entry": torch.tensor(entry, dtype=torch.int64, device=DEV), "heads": (hq, hkv, hd),
            "q": torch.zeros(rows, hq, hd, dtype=dt, device=DEV), "k": _randn((n_blocks, hkv, BLOCK, hd), g, dt),
            "v": _randn((n_blocks, hkv, hd, BLOCK), g, dt)}


def _cache(case, seed):
    hq, hkv, hd = HEADS[case["model"]]
    cached, new = _layout(case)
    n_blocks = _blocks_needed(cached, new, case["prefix"]) + 3
    perm = np.random.default_rng(seed).permutation(n_blocks).astype(np.int32)
    pre, table = _tables_host(cached, new, case["prefix"], perm)
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    kc = _randn((n_blocks, hkv, BLOCK, hd), g, dt)
    vc = _randn((n_blocks, hkv, hd, BLOCK), g, dt)
    rows = sum(new) + case.get("pad", 0)
    q = _randn((rows, hq, hd), g, dt)
    return {"q": q, "out": torch.empty_like(q), "k": kc, "v": vc, "prefix_blocks": _i32(pre),
            "prefix_len": case["prefix"], "table": _i32(table), "hkv": hkv,
            "max_ctx": max(c + x for c, x in zip(cached, new))}, cached, new


def _prepare_decode(case, seed):
    st, cached, _ = _cache(case, seed)
    n, pad = len(cached), case["pad"]
    st["slot"] = _i32(np.concatenate([np.arange(n)[::-1], np.full(pad, -1)]))
    st["pos"] = _i32(np.concatenate([cached, np.full(pad, -1)]))
    return st


def _prepare_prefill(case, seed):
    st, cached, new = _cache(case, seed)
    st["start"] = _i32(np.concatenate([[0], np.cumsum(new)]))
    st["slot"] = _i32(np.arange(len(new))[::-1].copy())
    st["pos"] = _i32(cached)
    st["max_new"] = max(new)
    return st


def prepare(case, seed):
    st = {"tables": _prepare_tables, "append": _prepare_append, "decode": _prepare_decode,
          "prefill": _prepare_prefill}[case["kind"]](case, seed)
    st["kind"] = case["kind"]
    return st


# ------------------------------------------------------------------ the plain forms

def _plain_tables(st):
    dev, (n_slots, wide) = st["table"].device, st["table"].shape
    prefix, first = st["prefix_len"], st["first"]
    cached, lengths, slot = st["cached"].long(), st["lengths"].long(), st["slot"].long()
    new = (lengths - cached).clamp(min=0)
    zero = torch.zeros(1, dtype=torch.int64, device=dev)
    seq_start = torch.cat([zero, new.cumsum(0)])
    have = torch.where(cached > prefix, (cached + BLOCK - 1) // BLOCK, torch.full_like(cached, first))
    need = ((lengths + BLOCK - 1) // BLOCK).clamp(max=wide)
    free_start = torch.cat([zero, (need - have).clamp(min=0).cumsum(0)]) + st["head"].long()
    b = torch.arange(wide, device=dev)[None, :]
    at = free_start[:-1, None] + b - have[:, None]
    n_free, pre, none = st["free"].numel(), st["prefix_blocks"], torch.full((), -1, dtype=torch.int32, device=dev)
    fresh = torch.where(at < n_free, st["free"][at.clamp(0, n_free - 1)], none)
    before = st["table"][slot]
    row = torch.where((b >= have[:, None]) & (b < need[:, None]), fresh, before)
    whole = (b < first) & (b < need[:, None])
    st["table"][slot] = torch.where(whole, pre[b.clamp(max=pre.numel() - 1)], row)
    st["seq_start"].copy_(seq_start)
    st["free_start"].copy_(free_start)
    rows = torch.arange(st["row_pos"].numel(), device=dev)
    live = rows < seq_start[-1]
    j = torch.searchsorted(seq_start[1:].contiguous(), rows, right=True).clamp(max=new.numel() - 1)
    pos = cached[j] + rows - seq_start[j]
    col = (pos // BLOCK).clamp(max=wide - 1)
    block = torch.where(pos < prefix, pre[col.clamp(max=pre.numel() - 1)], st["table"][slot[j], col]).long()
    inside = live & (pos < wide * BLOCK) & (block >= 0)
    st["row_slot"].copy_(torch.where(live, slot[j], -1))
    st["row_pos"].copy_(torch.where(live, pos, -1))
    st["row_entry"].copy_(torch.where(inside, block * BLOCK + pos % BLOCK, -1))
    return [st["table"], st["seq_start"], st["free_start"], st["row_slot"], st["row_pos"], st["row_entry"]]


def _plain_append(st):
    hq, hkv, hd = st["heads"]
    x = st["qkv"].view(-1, hq + 2 * hkv, hd)
    live = (st["pos"] >= 0).nonzero()[:, 0]
    x, pos = x[live], st["pos"][live].long()
    cos, sin = st["cos"][pos][:, None, :], st["sin"][pos][:, None, :]
    a, b = x[:, :hq + hkv, :hd // 2], x[:, :hq + hkv, hd // 2:]
    r = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1).to(st["q"].dtype)
    st["q"][live] = r[:, :hq]
    entry = st["entry"][live]
    block, off = entry // BLOCK, entry % BLOCK
    st["k"][block, :, off] = r[:, hq:]
    st["v"][block, :, :, off] = x[:, hq + hkv:].to(st["v"].dtype)
    return [st["q"], st["k"], st["v"]]


def _prefix_kv(st):
    """The prefix's keys and values in 32 bits, [n_kv_heads, prefix, head_dim] each."""
    idx, p = st["prefix_blocks"].long(), st["prefix_len"]
    hkv, hd = st["k"].shape[1], st["k"].shape[3]
    k = st["k"][idx].float().permute(1, 0, 2, 3).reshape(hkv, -1, hd)[:, :p]
    v = st["v"][idx].float().permute(1, 0, 3, 2).reshape(hkv, -1, hd)[:, :p]
    return k, v


def _own_kv(st, slot):
    """Keys and values of the given slots from the first block on that is not
    all prefix, in 32 bits, [slots, n_kv_heads, length, head_dim] each, and their positions."""
    b0, b1 = st["prefix_len"] // BLOCK, -(-st["max_ctx"] // BLOCK)
    idx = st["table"][slot.clamp(min=0)][:, b0:b1].long().clamp(min=0)
    hkv, hd = st["k"].shape[1], st["k"].shape[3]
    k = st["k"][idx].float().permute(0, 2, 1, 3, 4).reshape(len(slot), hkv, -1, hd)
    v = st["v"][idx].float().permute(0, 2, 1, 4, 3).reshape(len(slot), hkv, -1, hd)
    return k, v, b0 * BLOCK + torch.arange(k.shape[2], device=k.device)


def _part(q, k, v, seen):
    """Maximum, sum and weighted values of softmax(q k^T / sqrt(hd)) over `seen` keys."""
    s = (q @ k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(q.shape[-1]))
    s = torch.where(seen, s, torch.full((), -math.inf, device=s.device))
    m = s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    e = torch.exp(s - m)
    return m, e.sum(-1, keepdim=True), e @ v


def _join(a, b, dtype):
    """Two parts over separate keys as one, divided by their sum and rounded; nothing seen gives 0."""
    m = torch.maximum(a[0], b[0])
    fa, fb = torch.exp(a[0] - m), torch.exp(b[0] - m)
    total = a[1] * fa + b[1] * fb
    o = (a[2] * fa + b[2] * fb) / torch.where(total > 0, total, torch.ones((), device=m.device))
    return o.to(dtype)


def _plain_attention(st, pos, q_own, pos_own, slots, back):
    """Both parts of every token (positions `pos`): the prefix for all packed
    tokens in one product a KV head, the own context sequence by sequence
    (padded: `q_own`, `pos_own`; `back` is each token's place there)."""
    q, hkv = st["q"], st["hkv"]
    rows, hq, hd = q.shape
    group = hq // hkv
    k, v = _prefix_kv(st)
    qp = q.float().view(rows, hkv, group, hd).permute(1, 0, 2, 3).reshape(hkv, rows * group, hd)
    limit = (pos + 1).repeat_interleave(group)[None, :, None]
    pre = _part(qp, k, v, torch.arange(k.shape[1], device=q.device) < limit)
    pre = [x.view(hkv, rows, group, -1).permute(1, 0, 2, 3) for x in pre]
    ko, vo, kpos = _own_kv(st, slots)
    n, new = pos_own.shape
    qo = q_own.float().view(n, new, hkv, group, hd).permute(0, 2, 1, 3, 4).reshape(n, hkv, new * group, hd)
    seen = (kpos >= st["prefix_len"]) & (kpos <= pos_own.repeat_interleave(group, dim=1)[:, None, :, None])
    part = _part(qo, ko, vo, seen)
    part = [x.view(n, hkv, new, group, -1).permute(0, 2, 1, 3, 4).reshape(n * new, hkv, group, -1)[back] for x in part]
    return _join(pre, part, q.dtype).reshape(rows, hq, hd)


def _plain_decode(st):
    pos = st["pos"].long()
    rows = torch.arange(len(pos), device=pos.device)
    st["out"].copy_(_plain_attention(st, pos, st["q"][:, None], pos[:, None], st["slot"].long(), rows))
    return st["out"]


def _plain_prefill(st):
    start, first = st["start"].long(), st["pos"].long()
    n, new = len(first), st["max_new"]
    rows = torch.arange(st["q"].shape[0], device=start.device)
    i = torch.arange(new, device=start.device)[None, :]
    take = (start[:-1, None] + i).clamp(max=len(rows) - 1)
    j = torch.searchsorted(start[1:].contiguous(), rows, right=True)
    at = rows - start[j]
    st["out"].copy_(_plain_attention(st, first[j] + at, st["q"][take], first[:, None] + i, st["slot"].long(),
                                     j * new + at))
    return st["out"]


# ------------------------------------------------------------------ the framework's calls

def _own_tables(lp, st):
    lp.op_block_tables(st["slot"], st["cached"], st["lengths"], st["prefix_blocks"], st["prefix_len"], st["free"],
                       st["head"], st["table"], st["seq_start"], st["free_start"], st["row_slot"], st["row_pos"],
                       st["row_entry"])
    return [st["table"], st["seq_start"], st["free_start"], st["row_slot"], st["row_pos"], st["row_entry"]]


def _own_append(lp, st):
    lp.op_qkv_append(st["qkv"], st["cos"], st["sin"], st["pos"], st["entry"], st["q"], st["k"], st["v"])
    return [st["q"], st["k"], st["v"]]


def _workspace(st, need):
    """The workspace that a program allocates once and keeps."""
    if "ws" not in st:
        st["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    return st["ws"]


def _own_decode(lp, st):
    rows, hq, hd = st["q"].shape
    if "ws" not in st:
        _workspace(st, lp.prefix_decode_attention_ws_bytes(rows, hq, st["hkv"], hd, st["prefix_len"], st["max_ctx"]))
    lp.op_prefix_decode_attention(st["q"], st["out"], st["k"], st["v"], st["prefix_blocks"], st["prefix_len"],
                                  st["table"], st["slot"], st["pos"], st["max_ctx"], st["ws"])
    return st["out"]


def _own_prefill(lp, st):
    rows, hq, hd = st["q"].shape
    if "ws" not in st:
        _workspace(st, lp.prefix_prefill_attention_ws_bytes(rows, hq, st["hkv"], hd, st["prefix_len"],
                                                            st["max_ctx"]))
    lp.op_prefix_prefill_attention(st["q"], st["out"], st["k"], st["v"], st["prefix_blocks"], st["prefix_len"],
                                   st["table"], st["start"], st["slot"], st["pos"], st["max_new"], st["max_ctx"],
                                   st["ws"])
    return st["out"]


def run(st):
    if own:
        from paper_2410_02425_amd import lp
        return {"tables": _own_tables, "append": _own_append, "decode": _own_decode,
                "prefill": _own_prefill}[st["kind"]](lp, st)
    return {"tables": _plain_tables, "append": _plain_append, "decode": _plain_decode,
            "prefill": _plain_prefill}[st["kind"]](st)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    cached, new = _layout(case)
    n, rows = len(cached), sum(new)
    kind, prefix = case["kind"], case.get("prefix", 0)
    if kind == "tables":
        wide = max(-(-(c + x) // BLOCK) for c, x in zip(cached, new)) + 2
        taken = sum(max(0, -(-(c + x) // BLOCK) - (-(-c // BLOCK) if c > prefix else prefix // BLOCK))
                    for c, x in zip(cached, new))
        filled = taken + n * (prefix // BLOCK)
        return {"bytes": 12 * n + 8 * (n + 1) + 4 * min(filled, n * wide) + 4 * taken + 4 * -(-prefix // BLOCK)
                + 16 * (rows + case["pad"]), "flops": 0}
    hq, hkv, hd = HEADS[case["model"]]
    size = 4 if case["dtype"] == "f32" else 2
    if kind == "append":
        width = (hq + 2 * hkv) * hd
        return {"bytes": rows * (width * (4 + size) + 12) + 4 * rows * hd, "flops": 3 * rows * (hq + hkv) * hd}
    own_ctx = sum(c + x - prefix for c, x in zip(cached, new))
    seen = sum(c * x + x * (x + 1) // 2 for c, x in zip(cached, new))  # keys of all rows
    return {"bytes": ((prefix + own_ctx) * 2 * hkv * hd + 2 * rows * hq * hd) * size, "flops": 4 * seen * hq * hd}


# ------------------------------------------------------------------ the definitions in 64 bits

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
    where = st["entry"][keep]
    for h in range(hkv):
        k[:, h][where // BLOCK, where % BLOCK] = r[:, hq + h]
        v[:, h][where // BLOCK, :, where % BLOCK] = x[keep, hq + hkv + h]
    return [q, k, v]


def _exact_rows(st, rows, positions, slot, out):
    """softmax over positions 0..p for the given packed rows of one sequence, KV head by KV head, into `out`."""
    prefix, top = st["prefix_len"], max(positions) + 1
    blocks = [(st["prefix_blocks"], range(0, min(prefix, top))), (st["table"][slot], range(prefix, top))]
    where = torch.cat([b.long()[torch.tensor(list(p), dtype=torch.int64, device=DEV) // BLOCK] for b, p in blocks
                       if len(p)])
    off = torch.arange(top, device=DEV) % BLOCK
    hq, hkv = st["q"].shape[1], st["hkv"]
    group = hq // hkv
    ahead = torch.arange(top, device=DEV)[None, :] > torch.tensor(positions, device=DEV)[:, None]
    for h in range(hkv):
        k = st["k"][where, h, off].double()
        v = st["v"][where, h, :, off].double()
        for i in range(h * group, (h + 1) * group):
            s = st["q"][rows, i].double() @ k.T / math.sqrt(k.shape[1])
            out[rows, i] = torch.softmax(s.masked_fill(ahead, -math.inf), dim=1) @ v


def _exact_attention(case, seed):
    st = prepare(case, seed)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    slots, pos = st["slot"].tolist(), st["pos"].tolist()
    if case["kind"] == "decode":
        for m, (s, p) in enumerate(zip(slots, pos)):
            if p >= 0:
                _exact_rows(st, [m], [p], s, out)
    else:
        at = st["start"].tolist()
        for j, (s, p) in enumerate(zip(slots, pos)):
            n = at[j + 1] - at[j]
            if n:
                _exact_rows(st, list(range(at[j], at[j] + n)), list(range(p, p + n)), s, out)
    return out


def exact(case, seed):
    if case["kind"] == "tables":
        return None  # whole numbers
    if case["kind"] == "append":
        return _exact_append(case, seed)
    return _exact_attention(case, seed)
