"""Serving a batch that shares a prefix (include/lp_ops.h, last section): block
tables and cache entries from lengths, the QKV projection into the cache, and
decode and prefill attention over prefix and own blocks, against plain float64
implementations.  Every cache entry that no row may read is NaN."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_device_code as device_code
from oracle import transformer as T
from paper_2410_02425_amd import lp

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step at 1
gpu = pytest.mark.gpu


def ceil64(n):
    return -(-n // 64)


def i32(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


def values(rng, shape, dtype, scale=1.0):
    """Random values that dtype holds exactly, as float64."""
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(TYPES[dtype]).double().numpy()


# ------------------------------------------------------------------ block tables

def tables_reference(slot, cached, lengths, pre, P, free, head, table, max_rows):
    """The step's tables sequence by sequence, from the definition."""
    table, (n_slots, wide), F = table.copy(), table.shape, P // 64
    seq_start, free_start, at = [0], [head], head
    rows = []
    take_at = lambda i: free[i] if 0 <= i < len(free) else -1
    for s, c, n in zip(slot, cached, lengths):
        c, n = max(c, 0), max(n, 0)
        have, need = (ceil64(c) if c > P else F), min(ceil64(n) if n > P else min(ceil64(n), F), wide)
        new = max(0, n - c)
        own = {b: take_at(at + b - have) for b in range(have, need)}
        if 0 <= s < n_slots:
            for b in range(min(F, need)):
                table[s, b] = pre[b]
            for b, i in own.items():
                table[s, b] = i
        for p in range(c, c + min(new, max(0, max_rows - len(rows)))):
            b = p // 64
            if not 0 <= s < n_slots:
                i = -1
            elif p < P:
                i = pre[b]
            else:
                i = table[s, b] if b < wide else -1
            rows.append((s, p, i * 64 + p % 64 if i >= 0 else -1))
        at += len(own)
        seq_start.append(seq_start[-1] + new)
        free_start.append(at)
    rows += [(-1, -1, -1)] * (max_rows - len(rows))
    return table, seq_start, free_start, rows[:max_rows]


def run_tables(slot, cached, lengths, pre, P, free, head, table, max_rows, in_place=False):
    n = len(slot)
    t = i32(table)
    seq_start, free_start = i32([-7] * (n + 1)), i32([-7] * (n + 1))
    row_slot, row_pos = i32([-7] * max_rows), i32([-7] * max_rows)
    row_entry = torch.full((max_rows,), -7, dtype=torch.int64, device=DEV)
    head_t = i32([head])
    if in_place:
        free_start[n] = head
        head_t = free_start[n:]
    lp.op_block_tables(i32(slot), i32(cached), i32(lengths), i32(pre) if len(pre) else None, P, i32(free), head_t, t,
                       seq_start, free_start, row_slot, row_pos, row_entry)
    torch.cuda.synchronize()
    rows = list(zip(row_slot.tolist(), row_pos.tolist(), row_entry.tolist()))
    return t.cpu().numpy(), seq_start.tolist(), free_start.tolist(), rows


TABLE_CASES = [
    # sequences, prefix, cached range (past the prefix), new range, padding rows, free blocks beyond the need
    (1, 0, (0, 1), (1, 2), 0, 5), (1, 0, (0, 1), (0, 1), 3, 5), (1, 64, (0, 1), (65, 66), 1, 0),
    (4, 100, (0, 200), (1, 2), 0, 9), (64, 1024, (1, 700), (1, 2), 0, 3), (7, 63, (0, 3), (0, 200), 40, 3),
    (33, 640, (0, 1), (0, 500), 5, -10), (3, 65, (0, 130), (300, 900), 0, -4), (200, 0, (0, 90), (0, 70), 0, 1),
    (1030, 130, (0, 60), (0, 9), 77, 2), (2100, 64, (0, 100), (1, 2), 0, 0), (2, 5000, (0, 50), (4000, 9000), 9, 2),
]


@gpu
@pytest.mark.parametrize("n,P,cached,new,pad,spare", TABLE_CASES)
def test_block_tables(n, P, cached, new, pad, spare):
    rng = np.random.default_rng(n * 1000 + P)
    c = P + rng.integers(*cached, size=n)
    x = rng.integers(*new, size=n)
    slot = rng.permutation(n + 3)[:n]
    ends = c + x
    wide = int(max(ceil64(int(e)) for e in ends)) + 1
    perm = rng.permutation(ceil64(P) + n * wide + 200)
    pre = perm[:ceil64(P)]
    table = np.full((n + 3, wide), -1)
    at = ceil64(P)
    for s, k in zip(slot, c):
        if k > P:
            own = ceil64(int(k)) - P // 64
            table[s, :P // 64] = pre[:P // 64]
            table[s, P // 64:P // 64 + own] = perm[at:at + own]
            at += own
    need = sum(max(0, ceil64(int(e)) - (ceil64(int(k)) if k > P else P // 64)) for k, e in zip(c, ends) if e > P)
    free = perm[at:at + max(1, need + spare + 2)]
    max_rows = int(x.sum()) + pad
    args = (slot.tolist(), c.tolist(), ends.tolist(), pre, P, free, 2, table, max_rows)
    want = tables_reference(*args)
    for in_place in (False, True):
        got = run_tables(*args, in_place=in_place)
        assert np.array_equal(got[0], want[0])
        assert got[1] == want[1] and got[2] == want[2]
        assert got[3] == want[3]


@gpu
def test_block_tables_of_odd_data():
    """Slots outside the table, lengths below the cached ones, negative ones,
    lengths past the table's width, a prefix that a request computes itself,
    fewer row places than rows, a head outside the list: nothing is written
    outside the arrays, and what remains is as defined."""
    table = np.arange(5 * 4).reshape(5, 4) + 500
    args = ([0, 9, -1, 3, 1, 4], [0, 0, 10, 200, -5, 70], [100, 70, 30, 150, 3, 1000], [7, 8], 100,
            [40, 41, 42, 43, 44, 45, 46, 47], 1, table)
    for max_rows in (0, 1, 150, 1100, 1300):
        want = tables_reference(*args, max_rows)
        got = run_tables(*args, max_rows)
        assert np.array_equal(got[0], want[0]) and got[1:] == tuple(want[1:])
    for head in (-3, 8, 2 ** 31 - 1):
        a = args[:6] + (head, table)
        want, got = tables_reference(*a, 64), run_tables(*a, 64)
        assert np.array_equal(got[0], want[0]) and got[3] == want[3]
        assert got[2] == [min(x, 2 ** 31 - 1) for x in want[2]]


# ------------------------------------------------------------------ QKV append

def rope_tables(n_pos, hd):
    c, s = T.rope_cos_sin(np.arange(n_pos), hd, 10000.0)
    return c.astype(np.float32), s.astype(np.float32)


APPEND_CASES = [
    # dtype, Hq, Hkv, hd, positions of each run of rows, columns past the projection's
    ("f16", 32, 8, 128, [(0, 1)], 0), ("bf16", 32, 8, 128, [(5, 1)] * 3 + [(63, 1), (64, 1)], 0),
    ("f16", 8, 2, 64, [(0, 200), (61, 9)], 0), ("bf16", 6, 2, 128, [(3, 130), (250, 70)], 6),
    ("f32", 4, 4, 64, [(0, 37), (64, 64)], 0), ("f32", 5, 1, 128, [(1, 63), (127, 2)], 2),
    ("f16", 40, 40, 128, [(30, 70)], 2), ("f16", 3, 3, 64, [(7, 8), (0, 8), (56, 16)], 0),
    # V in 64-row tiles, whole blocks and ragged ones
    ("bf16", 64, 64, 64, [(0, 256), (7, 200)], 0), ("f16", 96, 96, 128, [(3, 333)], 2), ("f32", 64, 64, 64, [(64, 450)], 0),
]


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,runs,extra", APPEND_CASES)
def test_qkv_append(dtype, Hq, Hkv, hd, runs, extra):
    """Runs of consecutive positions, each in blocks of its own, with rows
    between them that have no position, a position past the tables or no entry;
    what no row names stays as it was."""
    rng = np.random.default_rng(Hq * 7 + len(runs))
    n_pos = max(p + n for p, n in runs)
    n_blocks = sum(ceil64(p + n) for p, n in runs) + 2
    blocks = rng.permutation(n_blocks)[: n_blocks - 2]
    pos, entry, at = [], [], 0
    for p, n in runs:
        k = np.arange(p, p + n)
        pos += k.tolist() + [-1, n_pos, p]
        entry += (blocks[at + k // 64] * 64 + k % 64).tolist() + [5, 9, [-1, n_blocks * 64, 2 ** 40][at % 3]]
        at += ceil64(p + n)
    rows, width = len(pos), (Hq + 2 * Hkv) * hd
    x = rng.standard_normal((rows, width + extra)).astype(np.float32)
    cos, sin = rope_tables(n_pos, hd)
    tdt = TYPES[dtype]
    q = torch.full((rows, Hq, hd), 7.0, dtype=tdt, device=DEV)
    kc = torch.full((n_blocks, Hkv, 64, hd), 7.0, dtype=tdt, device=DEV)
    vc = torch.full((n_blocks, Hkv, hd, 64), 7.0, dtype=tdt, device=DEV)
    xd = torch.from_numpy(x).to(DEV)[:, :width]
    lp.op_qkv_append(xd, torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV), i32(pos),
                     torch.tensor(entry, dtype=torch.int64, device=DEV), q, kc, vc)
    torch.cuda.synchronize()
    h = x[:, :width].astype(np.float64).reshape(rows, Hq + 2 * Hkv, hd)
    wq, wk, wv = np.full(q.shape, 7.0), np.full(kc.shape, 7.0), np.full(vc.shape, 7.0)
    size = np.zeros(q.shape), np.zeros(kc.shape)
    for r, (p, e) in enumerate(zip(pos, entry)):
        if not 0 <= p < n_pos:
            continue
        c, s = cos[p].astype(np.float64), sin[p].astype(np.float64)
        a, b = h[r, :Hq + Hkv, :hd // 2], h[r, :Hq + Hkv, hd // 2:]
        y = np.concatenate([a * c - b * s, b * c + a * s], axis=1)
        mag = np.concatenate([abs(a * c) + abs(b * s), abs(b * c) + abs(a * s)], axis=1)
        wq[r], size[0][r] = y[:Hq], mag[:Hq]
        if 0 <= e < n_blocks * 64:
            wk[e // 64, :, e % 64], size[1][e // 64, :, e % 64] = y[Hq:], mag[Hq:]
            wv[e // 64, :, :, e % 64] = h[r, Hq + Hkv:]
    u = UNIT[dtype]
    # the rotation is one rounded product and one fused step in fp32 (2^-24 of
    # the terms each), then one rounding to dtype (f16: at least 2^-25)
    for got, want, mag in ((q, wq, size[0]), (kc, wk, size[1]), (vc, wv, 0.0)):
        err = np.abs(got.double().cpu().numpy() - want)
        assert np.all(err <= (u if dtype != "f32" else 0) * np.abs(want) * (1 + 2 ** -10) + 2.0 ** -23 * mag + 2.0 ** -25)


# ------------------------------------------------------------------ attention

class Batch:
    """Sequences (their context lengths) over a prefix of P positions: K and V
    per sequence on the host, a cache that is NaN wherever no sequence has an
    entry, table rows in shuffled slots."""

    def __init__(self, rng, dtype, Hkv, hd, P, ctx, spare_slots=2, scale=1.0):
        own = [max(0, ceil64(c) - P // 64) if c > P else 0 for c in ctx]
        nP, n_slots = ceil64(P), len(ctx) + spare_slots
        self.n_blocks = nP + sum(own) + 3
        perm = rng.permutation(self.n_blocks)
        self.pre = perm[:nP]
        self.P, self.Hkv, self.hd, self.dtype, self.ctx = P, Hkv, hd, dtype, ctx
        kc = np.full((self.n_blocks, Hkv, 64, hd), np.nan)
        vc = np.full((self.n_blocks, Hkv, hd, 64), np.nan)
        pk, pv = values(rng, (P, Hkv, hd), dtype, scale), values(rng, (P, Hkv, hd), dtype)
        self.table = np.full((n_slots, max([P // 64 + o for o in own] + [1]) + 1), -1)
        self.slot = rng.permutation(n_slots)[:len(ctx)]

        def store(block_of, pos, k, v):
            for p, kk, vv in zip(pos, k, v):
                kc[block_of(p), :, p % 64], vc[block_of(p), :, :, p % 64] = kk, vv

        store(lambda p: self.pre[p // 64], range(P), pk, pv)
        at, self.K, self.V = nP, [], []
        for s, c, o in zip(self.slot, ctx, own):
            self.table[s, :P // 64] = self.pre[:P // 64]
            self.table[s, P // 64:P // 64 + o] = perm[at:at + o]
            at += o
            n = max(0, c - P)
            k, v = values(rng, (n, Hkv, hd), dtype, scale), values(rng, (n, Hkv, hd), dtype)
            store(lambda p: self.table[s, p // 64], range(P, P + n), k, v)
            self.K.append(np.concatenate([pk, k])[:c])
            self.V.append(np.concatenate([pv, v])[:c])
        self.kc = torch.from_numpy(kc).to(TYPES[dtype]).to(DEV)
        self.vc = torch.from_numpy(vc).to(TYPES[dtype]).to(DEV)
        self.pre_t = i32(self.pre) if P else None

    def reference(self, q, j, positions):
        """Attention of rows q of sequence j at these positions, and its error bound."""
        K, V = self.K[j], self.V[j]
        n = max(positions) + 1
        ref = T.attention(q, K[:n], V[:n], positions, np.arange(n), self.Hkv)
        mag = T.attention(q, K[:n], np.abs(V[:n]), positions, np.arange(n), self.Hkv)
        return ref, bound(self.dtype, q, K[:n], V[:n], ref, mag)


def bound(dtype, q, K, V, ref, mag):
    """Error of softmax(q K^T / sqrt(hd)) V with fp32 scores and sums: a score
    of hd products is off by (hd + 3) 2^-24 of its terms' sizes, which moves
    numerator and denominator; exp, the sums over n keys and the joins of parts
    add (n + 64) 2^-24; 16-bit kernels round each weight (u, at least 2^-25 in
    f16: n of them against a sum of at least 1) and the result (u)."""
    n, Hkv, hd = K.shape
    terms = np.linalg.norm(q, axis=-1).max() * np.linalg.norm(K, axis=-1).max() / np.sqrt(hd)
    tol = (2 * (hd + 3) * 2.0 ** -24 * terms + (n + 64) * 2.0 ** -24) * mag
    if dtype == "f32":
        return tol + 2.0 ** -24 * np.abs(ref)
    u = UNIT[dtype]
    small = n * 2.0 ** -25 * np.abs(V).max() if dtype == "f16" else 0.0
    return tol + u * (mag + np.abs(ref)) * (1 + 2.0 ** -6) + small + 2.0 ** -25


def run_decode(b, q, rows, Hq, max_ctx=None, slots=None, stream=None):
    """rows: (sequence, position) of each row; position -1: none."""
    M = len(rows)
    slot = i32([b.slot[j] for j, _ in rows]) if slots is None else i32(slots)
    pos = i32([p for _, p in rows])
    max_ctx = max_ctx or max([p for _, p in rows] + [0]) + 1
    out = torch.full((M, Hq, b.hd), float("nan"), dtype=TYPES[b.dtype], device=DEV)
    qd = torch.from_numpy(q).to(TYPES[b.dtype]).to(DEV)
    need = lp.prefix_decode_attention_ws_bytes(M, Hq, b.Hkv, b.hd, b.P, max_ctx)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    lp.op_prefix_decode_attention(qd, out, b.kc, b.vc, b.pre_t, b.P, i32(b.table), slot, pos, max_ctx, ws[:need])
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all()
    return out.double().cpu().numpy()


DECODE_CASES = [
    # dtype, Hq, Hkv, hd, prefix, contexts (at or below the prefix: rows inside it; 0: an empty row)
    ("f16", 4, 1, 128, 553, [613]), ("bf16", 32, 8, 128, 64, [65, 64, 63, 1, 0, 130]),
    ("f16", 32, 8, 128, 2000, [2001 + 37 * i for i in range(20)]),
    ("f16", 8, 8, 128, 100, [101, 100, 99, 400, 128, 129]), ("bf16", 40, 40, 128, 65, [66, 200, 65, 800]),
    ("f16", 64, 8, 128, 1000, [1000 + 9 * i for i in range(70)]), ("f16", 8, 8, 64, 0, [1, 64, 65, 0, 300]),
    ("bf16", 6, 2, 64, 1, [1, 2, 64, 65]), ("f16", 5, 1, 128, 200, [201, 260, 7]), ("bf16", 16, 1, 64, 320, [321] * 9),
    ("f16", 24, 1, 128, 191, [192, 700]), ("f32", 4, 4, 64, 100, [101, 130, 90, 0, 300]),
    ("f32", 8, 2, 128, 64, [64, 65, 500]), ("f32", 3, 1, 64, 0, [1, 77]), ("f32", 40, 8, 128, 700, [701 + i for i in range(30)]),
    ("f16", 32, 8, 128, 0, [600, 5, 64]), ("bf16", 8, 2, 128, 5000, [5001, 5300, 4000]),
    ("f16", 32, 8, 128, 64, [65 + i for i in range(130)]),
]


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,P,ctx", DECODE_CASES)
def test_prefix_decode_attention(dtype, Hq, Hkv, hd, P, ctx):
    rng = np.random.default_rng(P * 31 + len(ctx) + Hq)
    b = Batch(rng, dtype, Hkv, hd, P, ctx)
    q = values(rng, (len(ctx), Hq, hd), dtype)
    got = run_decode(b, q, [(j, c - 1) for j, c in enumerate(ctx)], Hq)
    for j, c in enumerate(ctx):
        if c == 0:
            assert np.all(got[j] == 0), j
            continue
        ref, tol = b.reference(q[j:j + 1], j, [c - 1])
        assert np.all(np.abs(got[j:j + 1] - ref) <= tol), (j, c, np.nanmax(np.abs(got[j] - ref) / tol))


def run_prefill(b, q, seqs, Hq, max_ctx=None, max_new=None, start=0, tail=0, slots=None):
    """seqs: (sequence, first position, rows); `start` and `tail` rows of q belong to none."""
    n = [x for _, _, x in seqs]
    rows = start + sum(n) + tail
    assert q.shape[0] == rows
    seq_start = i32(start + np.concatenate([[0], np.cumsum(n)]))
    max_ctx = max_ctx or max(p + x for _, p, x in seqs)
    max_new = max_new or max(n)
    out = torch.full((rows, Hq, b.hd), 7.0, dtype=TYPES[b.dtype], device=DEV)
    qd = torch.from_numpy(q).to(TYPES[b.dtype]).to(DEV)
    need = lp.prefix_prefill_attention_ws_bytes(rows, Hq, b.Hkv, b.hd, b.P, max_ctx)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    slot = i32([b.slot[j] for j, _, _ in seqs]) if slots is None else i32(slots)
    lp.op_prefix_prefill_attention(qd, out, b.kc, b.vc, b.pre_t, b.P, i32(b.table), seq_start, slot,
                                   i32([p for _, p, _ in seqs]), max_new, max_ctx, ws[:need])
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all()
    return out.double().cpu().numpy()


PREFILL_CASES = [
    # dtype, Hq, Hkv, hd, prefix, (first position past the prefix, or before it; new rows) of each sequence
    ("f16", 32, 8, 128, 500, [(0, 20), (0, 1), (0, 33), (0, 64)]), ("bf16", 8, 2, 128, 64, [(0, 65), (30, 7), (-64, 64)]),
    ("f16", 8, 8, 128, 1000, [(0, 300)]), ("f16", 4, 4, 64, 100, [(0, 5), (-30, 60), (-100, 130), (77, 1)]),
    ("bf16", 40, 40, 128, 130, [(0, 30), (0, 129)]), ("f16", 64, 8, 128, 2048, [(0, 150), (500, 40)]),
    ("f16", 6, 2, 128, 1, [(0, 31), (0, 32), (0, 33)]), ("bf16", 5, 1, 64, 63, [(0, 70), (1, 1)]),
    ("f16", 32, 8, 128, 0, [(0, 200), (300, 50), (0, 1)]), ("f32", 4, 4, 64, 64, [(0, 20), (0, 1), (-64, 100)]),
    ("f32", 8, 2, 128, 100, [(0, 70), (-10, 5)]), ("f32", 6, 2, 64, 0, [(0, 65), (20, 3)]),
    ("bf16", 32, 8, 128, 300, [(0, 700), (0, 3)]), ("f16", 16, 2, 128, 4000, [(0, 3), (0, 9)]),
    ("f16", 8, 1, 64, 777, [(i % 5, 1 + i % 7) for i in range(70)]), ("bf16", 16, 16, 128, 640, [(0, 12)] * 11),
    ("f16", 8, 8, 64, 40, [(2500, 130), (0, 2)]),
    # few tiles over long contexts of their own, beside rows that have none
    ("f32", 4, 2, 64, 70, [(1500, 30), (0, 40), (-70, 10), (-30, 1)]), ("bf16", 8, 1, 128, 500, [(-500, 20), (3000, 9), (0, 1)]),
    ("f16", 4, 4, 128, 0, [(0, 1), (1300, 64), (0, 0), (0, 300)]),
]


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,P,seqs", PREFILL_CASES)
def test_prefix_prefill_attention(dtype, Hq, Hkv, hd, P, seqs):
    rng = np.random.default_rng(P * 17 + len(seqs) + Hq)
    b = Batch(rng, dtype, Hkv, hd, P, [max(P + c + n, 0) for c, n in seqs])
    rows = 3 + sum(n for _, n in seqs) + 2
    q = values(rng, (rows, Hq, hd), dtype)
    got = run_prefill(b, q, [(j, P + c, n) for j, (c, n) in enumerate(seqs)], Hq, start=3, tail=2)
    assert np.all(got[:3] == 7) and np.all(got[-2:] == 7)     # rows of no sequence
    r = 3
    for j, (c, n) in enumerate(seqs):
        if n == 0:      # no row to look at
            continue
        pos = np.arange(P + c, P + c + n)
        ref, tol = b.reference(q[r:r + n], j, pos)
        err = np.abs(got[r:r + n] - ref)
        assert np.all(err <= tol), (j, np.nanmax(err / tol))
        r += n


@gpu
@pytest.mark.parametrize("dtype,hd", [("f16", 128), ("bf16", 64), ("f32", 64)])
def test_attention_of_missing_blocks_slots_and_positions(dtype, hd):
    """Missing blocks (-1 and past the pool) are left out of a row's keys, in the
    prefix and in its own; slots outside the table and negative positions give
    zeros; contexts are clamped to max_ctx."""
    rng = np.random.default_rng(5)
    Hq, Hkv, P = 8, 2, 200
    b = Batch(rng, dtype, Hkv, hd, P, [500, 300, 260, 210, 150])
    b.pre[1] = -1
    b.table[b.slot[0], 5] = b.n_blocks
    b.table[b.slot[1], 3:] = -1
    b.pre_t = i32(b.pre)
    rows = [(0, 499), (1, 299), (2, 259), (3, -1), (3, 209), (4, 149), (2, 255)]
    q = values(rng, (len(rows), Hq, hd), dtype)
    slots = [b.slot[j] for j, _ in rows]
    slots[6] = b.table.shape[0]
    got = run_decode(b, q, rows, Hq, max_ctx=490, slots=slots)
    gone = {0: [(64, 128), (320, 384)], 1: [(64, 128), (200, 300)], 2: [(64, 128)], 3: [(64, 128)], 4: [(64, 128)]}
    seqs = [(0, 488, 4), (1, 290, 5), (4, 140, 10)]
    q2 = values(rng, (sum(x for _, _, x in seqs), Hq, hd), dtype)
    got2 = run_prefill(b, q2, seqs, Hq, max_ctx=490, slots=[b.slot[0], b.slot[1], -1])

    def check(qr, have, j, p):
        keep = np.array([i for i in range(min(p + 1, 490)) if not any(lo <= i < hi for lo, hi in gone[j])])
        K, V = b.K[j][keep], b.V[j][keep]
        args = ([p], np.arange(len(keep)), Hkv)
        ref, mag = (T.attention(qr, K, v, *args) for v in (V, np.abs(V)))
        assert np.all(np.abs(have - ref) <= bound(dtype, qr, K, V, ref, mag)), (j, p)

    for m, (j, p) in enumerate(rows):
        if m in (3, 6):
            assert np.all(got[m] == 0)
        else:
            check(q[m:m + 1], got[m:m + 1], j, p)
    assert np.all(got2[9:] == 0)
    for r in range(9):
        j, p = (0, 488 + r) if r < 4 else (1, 290 + r - 4)
        check(q2[r:r + 1], got2[r:r + 1], j, p)


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd", [("f16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 64)])
def test_values_behind_a_row_do_not_reach_it(dtype, Hq, Hkv, hd):
    """Infinities and NaN in K and V at positions that later rows of the same
    sequence see: earlier rows keep their results, rows from there on get NaN."""
    rng = np.random.default_rng(6)
    P, n = 70, 150
    b = Batch(rng, dtype, Hkv, hd, P, [P + n, P + 40])
    q = values(rng, (P + n + 40, Hq, hd), dtype)
    seqs = [(0, 0, P + n), (1, P, 40)]                  # the first computes the prefix itself
    clean = run_prefill(b, q, seqs, Hq)
    bad = P + 37
    blk, off = b.table[b.slot[0], bad // 64], bad % 64
    b.kc[blk, 0, off] = float("nan")
    b.vc[blk, :, :, off] = float("inf")
    got = run_prefill(b, q, seqs, Hq)
    assert np.array_equal(got[:bad], clean[:bad]) and np.array_equal(got[P + n:], clean[P + n:])
    assert np.isnan(got[bad:P + n, :Hq // Hkv]).all()             # NaN scores
    assert not np.isfinite(got[bad:P + n, Hq // Hkv:]).any()      # infinite values
    # the same inside the prefix, seen by rows of every sequence from there on
    blk, off = b.pre[0], 30
    b.vc[blk, :, :, off] = float("nan")
    got = run_prefill(b, q, seqs, Hq)
    assert np.array_equal(got[:30], clean[:30]) and np.isnan(got[30:]).all()
    rows = [(0, 12), (0, 29), (0, 30), (1, P + 5)]
    dec = run_decode(b, q[:4], rows, Hq)
    for m, (j, p) in enumerate(rows[:2]):
        ref, tol = b.reference(q[m:m + 1], j, [p])
        assert np.all(np.abs(dec[m:m + 1] - ref) <= tol)
    assert np.isnan(dec[2:]).all()


@gpu
@pytest.mark.parametrize("dtype,lo,hi", [("f16", 2, 30), ("bf16", 2, 90), ("f32", 2, 90)])
def test_scores_of_any_size(dtype, lo, hi):
    """Scores from 2^lo to 2^hi, one size a head, each exact in fp32: the weight
    of the largest stays 1, whichever part it is in."""
    rng = np.random.default_rng(hi)
    Hq = Hkv = 8
    hd, P = 64, 130
    ctx = [131, 200, 420, 130]
    b = Batch(rng, dtype, Hkv, hd, P, ctx)
    e = np.linspace(lo, hi - 6, Hkv).astype(int)              # 64 dims add 6 bits
    q = np.broadcast_to((2.0 ** (e // 2))[None, :, None], (4, Hq, hd)).copy()
    pre = rng.integers(64, 128, (P, Hkv)) * rng.choice([-1.0, 1.0], (P, Hkv))
    for j, c in enumerate(ctx):
        own = rng.integers(64, 128, (max(0, c - P), Hkv)) * rng.choice([-1.0, 1.0], (max(0, c - P), Hkv))
        k = np.concatenate([pre, own])[:c] * 2.0 ** (e - e // 2 - 6)
        b.K[j] = np.repeat(k[:, :, None], hd, axis=2)
        for p in range(c):
            blk = b.pre[p // 64] if p < P else b.table[b.slot[j], p // 64]
            b.kc[blk, :, p % 64] = torch.from_numpy(b.K[j][p]).to(b.kc.dtype).to(DEV)
    assert torch.isfinite(torch.from_numpy(q).to(TYPES[dtype])).all()
    got = run_decode(b, q, [(j, c - 1) for j, c in enumerate(ctx)], Hq)
    u = UNIT[dtype]
    for j, c in enumerate(ctx):
        args = ([c - 1], np.arange(c), Hkv)
        ref, mag = (T.attention(q[j:j + 1], b.K[j], v, *args) for v in (b.V[j], np.abs(b.V[j])))
        # the scores are exact: only weights, sums and the result are rounded
        tol = ((c + 64) * 2.0 ** -24 + (u if dtype != "f32" else 0)) * (mag + np.abs(ref)) * 1.02 + 2.0 ** -24
        # the scale 1/8 is exact, its base-2 factor is not: 2^-23 of a score's distance from the largest,
        # which weights that are not yet 0 keep below 2^7
        assert np.all(np.abs(got[j:j + 1] - ref) <= tol + 2.0 ** -15 * mag), j


@gpu
@pytest.mark.parametrize("P,rows,Hq", [(8192, 3, 1), (0, 260, 64)])
def test_sums_over_many_large_scores_meet_at_one_maximum(P, rows, Hq):
    """Scores of 4,000 in base 2, with values of 1 at the first 8,192 positions
    and -1 at the others: an error of one part's (or, in a walk of one part, of
    one block's) sums against another's is the result's.  Every block holds its
    half's largest score, and the halves' largest are such that score times
    log2(e) / sqrt(64), rounded in fp32, is off by 2^-13 up in one, down in the other."""
    rng = np.random.default_rng(1)
    hd, n, top = 64, 16384, (31.671875, 31.875)
    x = [np.minimum(rng.integers(0, 2048, 8192) / 64, t) for t in top]
    for half, t in zip(x, top):
        half[rng.integers(0, 64, 128) + 64 * np.arange(128)] = t
    score = 22144 + np.concatenate(x)                # 128 * 173 + ..: exact in f16 as two products, and in fp32
    kc = torch.zeros(256, 1, 64, hd, dtype=torch.float16, device=DEV)
    kc[..., 0] = 173
    kc[:, 0, :, 1] = torch.from_numpy(score - 22144).half().view(256, 64).to(DEV)
    assert torch.equal(kc[:, 0, :, 1].double().cpu().flatten(), torch.from_numpy(score - 22144))
    v = np.where(np.arange(n) < 8192, 1.0, -1.0)
    vc = torch.from_numpy(v).half().view(256, 1, 1, 64).expand(256, 1, hd, 64).contiguous().to(DEV)
    q = torch.zeros(rows, Hq, hd, dtype=torch.float16, device=DEV)
    q[..., 0], q[..., 1] = 128, 1
    out = torch.empty_like(q)
    table = i32([np.arange(256)])
    ws = torch.empty(lp.prefix_prefill_attention_ws_bytes(rows, Hq, 1, hd, P, n) + 16, dtype=torch.uint8, device=DEV)
    lp.op_prefix_prefill_attention(q, out, kc, vc, table[0, :P // 64].contiguous(), P, table, i32([0, rows]), i32([0]),
                                   i32([n - rows]), rows, n, ws)
    got = out.double().cpu().numpy()
    # weights are rounded to f16 against the largest of their own half, and the sums scaled to the row's
    weight = [np.exp((22144 + a - 22144 - t) / 8) for a, t in zip(x, top)]
    scale = np.repeat([np.exp((top[0] - top[1]) / 8), 1.0], 8192)
    held = torch.from_numpy(np.concatenate(weight)).half().double().numpy() * scale
    weight = np.concatenate(weight) * scale
    for r in range(rows):
        c = n - rows + r + 1
        ref = (held[:c] * v[:c]).sum() / weight[:c].sum()
        # two fp32 sums over n terms in random order: 2^-24 of each partial sum, in all 2^-24 sqrt(n / 3) = 4.4e-6
        # of the whole as a standard deviation, four of them; a weight next to a tie (6e-4 of them) may round the
        # other way: 6e-4 * 2^-11; the result's own rounding
        assert np.all(np.abs(got[r] - ref) <= 2.0 ** -11 * abs(ref) + 1.8e-5 + 3e-7), (r, got[r, 0, 0] - ref)


# ------------------------------------------------------------------ a step of all four

class Service:
    """A layer of requests behind one prefix, served by the four calls; K, V and
    q of every position come from random projections."""

    def __init__(self, rng, dtype, Hq, Hkv, hd, P, n, extra_blocks=40):
        self.rng, self.dtype, self.Hq, self.Hkv, self.hd, self.P, self.n = rng, dtype, Hq, Hkv, hd, P, n
        tdt = TYPES[dtype]
        n_blocks = ceil64(P) + extra_blocks
        perm = rng.permutation(n_blocks)
        self.pre, self.free = i32(perm[:ceil64(P)]), i32(perm[ceil64(P):])
        self.kc = torch.full((n_blocks, Hkv, 64, hd), float("nan"), dtype=tdt, device=DEV)
        self.vc = torch.full((n_blocks, Hkv, hd, 64), float("nan"), dtype=tdt, device=DEV)
        self.table = i32(np.full((n, ceil64(P) + 8), -1))
        self.cos, self.sin = (torch.from_numpy(x).to(DEV) for x in rope_tables(P + 400, hd))
        self.slot = i32(rng.permutation(n))
        self.head = i32([0])

    def tables(self, slot, cached, lengths, free_head, max_rows):
        n = slot.numel()
        st = dict(seq_start=torch.empty(n + 1, dtype=torch.int32, device=DEV),
                  free_start=torch.empty(n + 1, dtype=torch.int32, device=DEV),
                  row_slot=torch.empty(max_rows, dtype=torch.int32, device=DEV),
                  row_pos=torch.empty(max_rows, dtype=torch.int32, device=DEV),
                  row_entry=torch.empty(max_rows, dtype=torch.int64, device=DEV))
        lp.op_block_tables(slot, cached, lengths, self.pre, self.P, self.free, free_head, self.table, **st)
        return st

    def append(self, qkv, st):
        q = torch.zeros(qkv.shape[0], self.Hq, self.hd, dtype=TYPES[self.dtype], device=DEV)
        lp.op_qkv_append(qkv, self.cos, self.sin, st["row_pos"], st["row_entry"], q, self.kc, self.vc)
        return q

    def projection(self, rows):
        return torch.from_numpy(self.rng.standard_normal((rows, (self.Hq + 2 * self.Hkv) * self.hd)).astype(np.float32))

    def exact(self, qkv, pos):
        """Rotated q and k, and v, of projections at positions, rounded as the cache holds them."""
        x = qkv.double().numpy().reshape(len(pos), -1, self.hd)
        h = self.Hq + self.Hkv
        r = T.rope(x[:, :h], np.asarray(pos), 10000.0)
        hold = lambda a: torch.from_numpy(a).to(TYPES[self.dtype]).double().numpy()
        return hold(r[:, :self.Hq]), hold(r[:, self.Hq:]), hold(x[:, h:])


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,P", [("f16", 8, 2, 128, 150), ("bf16", 8, 8, 64, 64), ("f32", 4, 2, 64, 100)])
def test_a_service_from_tables_to_tokens(dtype, Hq, Hkv, hd, P):
    """The prefix computed once by a request of its own, then four requests
    admitted behind it and three decode steps, all four calls in turn."""
    rng = np.random.default_rng(P)
    n = 4
    s = Service(rng, dtype, Hq, Hkv, hd, P, n)
    tdt = TYPES[dtype]

    def prefill(slot, cached, new):
        """Tables, append and attention of a step; the host's q, k, v per sequence."""
        rows = int(sum(new))
        st = s.tables(slot, i32(cached), i32(np.asarray(cached) + new), s.head, rows + 3)
        s.head = st["free_start"][-1:]
        qkv = s.projection(rows + 3)
        q = s.append(qkv.to(DEV), st)
        out = torch.zeros_like(q)
        top = int(max(np.asarray(cached) + new))
        ws = torch.empty(lp.prefix_prefill_attention_ws_bytes(rows + 3, Hq, Hkv, hd, P, top) + 16, dtype=torch.uint8, device=DEV)
        lp.op_prefix_prefill_attention(q, out, s.kc, s.vc, s.pre, P, s.table, st["seq_start"], slot, i32(cached),
                                       int(max(new)), top, ws)
        torch.cuda.synchronize()
        parts, r = [], 0
        for c, x in zip(cached, new):
            parts.append((s.exact(qkv[r:r + x], range(c, c + x)), out[r:r + x].double().cpu().numpy(), c))
            r += x
        assert not out[rows:].any()
        return parts

    def check(got, q, K, V, pos):
        ref, mag = (T.attention(q, K, v, pos, np.arange(len(K)), Hkv) for v in (V, np.abs(V)))
        # q, k and v may each be off by a rounding of the cache's type where the
        # rotation in fp32 falls on the other side of a tie: counted as two steps of every product
        flip = 2 * UNIT[dtype] * np.linalg.norm(q, axis=-1).max() * np.linalg.norm(K, axis=-1).max() / np.sqrt(hd)
        tol = bound(dtype, q, K, V, ref, mag) + (2 * 2.0 ** -10 * flip + 2.0 ** -20) * mag
        assert np.all(np.abs(got - ref) <= tol), np.max(np.abs(got - ref) / tol)

    # one request computes the prefix: its rows go to the prefix's blocks
    (part,) = prefill(s.slot[:1], [0], [P])
    (q, pk, pv), got, _ = part
    check(got, q, pk, pv, np.arange(P))
    # all requests behind it
    new = [5, 64, 1, 33]
    K, V = [], []
    for (q, k, v), got, c in prefill(s.slot, [P] * n, new):
        K.append(np.concatenate([pk, k]))
        V.append(np.concatenate([pv, v]))
        check(got, q, K[-1], V[-1], np.arange(P, P + len(k)))
    # decode steps
    length = P + np.asarray(new)
    for step in range(3):
        st = s.tables(s.slot, i32(length), i32(length + 1), s.head, n)
        s.head = st["free_start"][-1:]
        qkv = s.projection(n)
        q = s.append(qkv.to(DEV), st)
        out = torch.empty_like(q)
        top = int(length.max()) + 1
        ws = torch.empty(lp.prefix_decode_attention_ws_bytes(n, Hq, Hkv, hd, P, top) + 16, dtype=torch.uint8, device=DEV)
        lp.op_prefix_decode_attention(q, out, s.kc, s.vc, s.pre, P, s.table, st["row_slot"], st["row_pos"], top, ws)
        torch.cuda.synchronize()
        for j in range(n):
            qj, k, v = s.exact(qkv[j:j + 1], [length[j]])
            K[j], V[j] = np.concatenate([K[j], k]), np.concatenate([V[j], v])
            check(out[j:j + 1].double().cpu().numpy(), qj, K[j], V[j], [int(length[j])])
        length = length + 1
    taken = sum(ceil64(int(x)) - P // 64 for x in length)
    assert s.head.item() == taken


@gpu
def test_whole_block_prefix_reads_as_an_ordinary_table():
    """With a prefix of whole blocks the table serves the attention calls
    without a prefix too: both agree within their bounds."""
    rng = np.random.default_rng(12)
    Hq, Hkv, hd, P, ctx = 8, 2, 128, 192, [193, 300, 450]
    b = Batch(rng, "f16", Hkv, hd, P, ctx)
    q = values(rng, (3, Hq, hd), "f16")
    got = run_decode(b, q, [(j, c - 1) for j, c in enumerate(ctx)], Hq)
    qd = torch.from_numpy(q).half().to(DEV)
    out = torch.empty_like(qd)
    ws = torch.empty(lp.decode_attention_ws_bytes(3, Hq, hd, 450), dtype=torch.uint8, device=DEV)
    lp.op_decode_attention(qd, out, b.kc, b.vc, i32(b.table), i32(b.slot), i32([c - 1 for c in ctx]), Hkv, 450, ws)
    other = out.double().cpu().numpy()
    for j, c in enumerate(ctx):
        ref, tol = b.reference(q[j:j + 1], j, [c - 1])
        assert np.all(np.abs(got[j:j + 1] - ref) <= tol) and np.all(np.abs(other[j:j + 1] - ref) <= tol)


@gpu
def test_decode_steps_in_a_captured_graph():
    """Tables (with the free list's head updated in place), append and decode
    attention captured once and replayed, with eager work between the replays,
    against the same steps run eagerly."""
    P, n, Hq, Hkv, hd, steps = 100, 5, 8, 2, 64, 5
    results = []
    for captured in (False, True):
        rng = np.random.default_rng(9)
        s = Service(rng, "f16", Hq, Hkv, hd, P, n)
        s.kc.normal_(generator=torch.Generator(DEV).manual_seed(1))
        s.vc.normal_(generator=torch.Generator(DEV).manual_seed(2))
        cached = i32([P + 20, P, P + 27, P + 63, P + 60])
        one = torch.ones_like(cached)
        lengths = cached + one
        for j in range(n):      # what each request holds before the first step
            have = ceil64(int(cached[j])) if int(cached[j]) > P else P // 64
            row = torch.arange(30 + 4 * j - P // 64, 30 + 4 * j - P // 64 + have, dtype=torch.int32, device=DEV)
            row[:P // 64] = s.pre[:P // 64]
            s.table[int(s.slot[j]), :have] = s.free[(row % s.free.numel()).long()]
        qkvs = [s.projection(n).to(DEV) for _ in range(steps)]
        qkv, top = torch.empty_like(qkvs[0]), P + 80
        st = dict(seq_start=i32([0] * (n + 1)), free_start=i32([0] * (n + 1)), row_slot=i32([0] * n), row_pos=i32([0] * n),
                  row_entry=torch.zeros(n, dtype=torch.int64, device=DEV))
        q = torch.zeros(n, Hq, hd, dtype=torch.float16, device=DEV)
        out = torch.zeros_like(q)
        ws = torch.empty(lp.prefix_decode_attention_ws_bytes(n, Hq, Hkv, hd, P, top), dtype=torch.uint8, device=DEV)

        def step():
            lp.op_block_tables(s.slot, cached, lengths, s.pre, P, s.free, st["free_start"][n:], s.table, **st)
            lp.op_qkv_append(qkv, s.cos, s.sin, st["row_pos"], st["row_entry"], q, s.kc, s.vc)
            lp.op_prefix_decode_attention(q, out, s.kc, s.vc, s.pre, P, s.table, st["row_slot"], st["row_pos"], top, ws)
            cached.add_(one)
            lengths.add_(one)

        if captured:
            torch.cuda.synchronize()
            graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            with torch.cuda.graph(graph, stream=side):
                step()
        seen = []
        for k in range(steps):
            qkv.copy_(qkvs[k])
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            seen.append([out.clone(), s.table.clone(), st["row_entry"].clone(), st["free_start"].clone()])
            torch.ones(1000, device=DEV).sum().item()          # the program's own eager work
        results.append(seen)
    for a, b in zip(*results):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
        assert torch.isfinite(a[0]).all()


@gpu
def test_two_streams_at_once():
    """The same calls on two streams with workspaces of their own, many times over, give what one gives alone."""
    rng = np.random.default_rng(3)
    Hq, Hkv, hd, P, ctx = 32, 8, 128, 700, [701 + 40 * i for i in range(16)]
    b = Batch(rng, "f16", Hkv, hd, P, ctx)
    q = [torch.from_numpy(values(rng, (16, Hq, hd), "f16")).half().to(DEV) for _ in range(2)]
    slot, pos, table, top = i32(b.slot), i32([c - 1 for c in ctx]), i32(b.table), max(ctx)
    nb = lp.prefix_decode_attention_ws_bytes(16, Hq, Hkv, hd, P, top)

    def call(k, out, ws):
        lp.op_prefix_decode_attention(q[k], out, b.kc, b.vc, b.pre_t, P, table, slot, pos, top, ws)

    wss = [torch.empty(nb, dtype=torch.uint8, device=DEV) for _ in range(2)]
    alone = [torch.empty_like(q[0]) for _ in range(2)]
    for k in range(2):
        call(k, alone[k], wss[k])
    outs = [[torch.empty_like(q[0]) for _ in range(10)] for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(10):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                call(k, outs[k][i], wss[k])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(o, alone[k]) for o in outs[k])


# ------------------------------------------------------------------ calls of other shapes

@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,n", [("f16", 8, 2, 128, 40), ("bf16", 16, 16, 64, 45), ("f32", 24, 1, 64, 12)])
def test_decode_batches_of_odd_rows(dtype, Hq, Hkv, hd, n):
    """Rows inside the prefix before and behind an infinite value, padding rows,
    the same slot twice, a max_ctx and a table far above any context."""
    rng = np.random.default_rng(n)
    P, bad = 700, 300
    ctx = [P + 1 + 29 * i for i in range(n)]
    b = Batch(rng, dtype, Hkv, hd, P, ctx)
    b.table = np.concatenate([b.table, np.full((b.table.shape[0], 1500), -1)], axis=1)
    rows = [(j, c - 1) for j, c in enumerate(ctx)]
    rows += [(0, -1), (1, 12), (1, bad - 1), (1, bad), (2, 64), (2, 64), (0, -5), (3, ctx[3] - 1), (3, 0), (4, P - 1)]
    q = values(rng, (len(rows), Hq, hd), dtype)

    def check(got, m):
        j, p = rows[m]
        ref, tol = b.reference(q[m:m + 1], j, [p])
        assert np.all(np.abs(got[m:m + 1] - ref) <= tol), (m, np.nanmax(np.abs(got[m:m + 1] - ref) / tol))

    b.clean = b.vc.clone()
    for top in (None, b.table.shape[1] * 64):
        got = run_decode(b, q, rows, Hq, max_ctx=top)
        for m, (_, p) in enumerate(rows):
            if p < 0:
                assert np.all(got[m] == 0)
            else:
                check(got, m)
        b.vc[int(b.pre[bad // 64]), :, :, bad % 64] = float("inf")
        got = run_decode(b, q, rows, Hq, max_ctx=top)
        for m, (_, p) in enumerate(rows):
            if p < 0:
                assert np.all(got[m] == 0)
            elif p < bad:
                check(got, m)
            else:
                assert not np.isfinite(got[m]).any()
        b.vc.copy_(b.clean)


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,P,seqs", [
    ("f16", 64, 64, 64, 130, [(0, 900), (-30, 100), (3, 0), (40, 17)]),
    ("bf16", 64, 8, 128, 70, [(0, 1), (0, 1000), (200, 90)]),
    ("f32", 8, 8, 64, 200, [(0, 150), (0, 0), (0, 0), (-200, 90)]),
])
def test_prefill_of_many_rows(dtype, Hq, Hkv, hd, P, seqs):
    """Batches whose tiles fill the GPU, with sequences that have no new row,
    infinite values behind some rows, and a max_ctx and max_new above any."""
    rng = np.random.default_rng(Hq + P)
    b = Batch(rng, dtype, Hkv, hd, P, [P + c + n for c, n in seqs])
    rows = 3 + sum(n for _, n in seqs) + 2
    q = values(rng, (rows, Hq, hd), dtype)
    calls = [(j, P + c, n) for j, (c, n) in enumerate(seqs)]
    got = run_prefill(b, q, calls, Hq, start=3, tail=2)
    big = run_prefill(b, q, calls, Hq, start=3, tail=2, max_ctx=b.table.shape[1] * 64, max_new=5000)
    for out in (got, big):
        assert np.all(out[:3] == 7) and np.all(out[-2:] == 7)
    # every 7th row and the last ones
    r, long = 3, max(range(len(seqs)), key=lambda j: seqs[j][1])
    for j, p, n in calls:
        some = np.unique(np.concatenate([np.arange(0, n, 7), np.arange(max(0, n - 3), n)])).astype(int)
        if n:
            ref, tol = b.reference(q[r:r + n][some], j, p + some)
            for out in (got, big):
                assert np.all(np.abs(out[r:r + n][some] - ref) <= tol), j
        if j == long:
            first = r
        r += n
    j, p, n = calls[long]
    at = p + n // 2
    blk = b.table[b.slot[j], at // 64] if at >= P else b.pre[at // 64]
    b.vc[int(blk), :, :, at % 64] = float("-inf")
    odd = run_prefill(b, q, calls, Hq, start=3, tail=2)
    behind = np.arange(first + n // 2, first + n)
    assert not np.isfinite(odd[behind]).any()
    before = np.setdiff1d(np.arange(rows), behind)
    assert np.array_equal(odd[before], got[before])


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd", [("f16", 8, 2, 128), ("bf16", 32, 2, 64), ("f32", 4, 2, 64)])
def test_rows_that_only_read_the_prefix(dtype, Hq, Hkv, hd):
    """No row has a block of its own: decode rows and prompts inside a prefix of two blocks, and of many."""
    rng = np.random.default_rng(hd + Hq)
    for P in (128, 1000):
        b = Batch(rng, dtype, Hkv, hd, P, [P, P, P])
        rows = [(m % 3, [-1, 0, P - 1, 63, 64, m % P][m % 6]) for m in range(140)]
        q = values(rng, (140, Hq, hd), dtype)
        got = run_decode(b, q, rows, Hq)
        for m, (j, p) in enumerate(rows):
            if p < 0:
                assert np.all(got[m] == 0)
            else:
                ref, tol = b.reference(q[m:m + 1], j, [p])
                assert np.all(np.abs(got[m:m + 1] - ref) <= tol), m
        seqs = [(0, 0, 70), (1, P - 30, 30), (2, 40, 37)]
        got = run_prefill(b, q, seqs, Hq, start=1, tail=2)
        assert np.all(got[:1] == 7) and np.all(got[-2:] == 7)
        r = 1
        for j, p, n in seqs:
            ref, tol = b.reference(q[r:r + n], j, np.arange(p, p + n))
            assert np.all(np.abs(got[r:r + n] - ref) <= tol), j
            r += n


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_of_a_padded_batch(dtype):
    """150 places for sequences of which five have rows, the others none and no slot."""
    rng = np.random.default_rng(150)
    P, Hq, Hkv, hd = 90, 8, 2, 64
    new = np.zeros(150, int)
    new[[3, 63, 64, 100, 149]] = [40, 1, 33, 70, 9]
    b = Batch(rng, dtype, Hkv, hd, P, [P + n for n in new])
    q = values(rng, (new.sum() + 4, Hq, hd), dtype)
    got = run_prefill(b, q, [(j, P, n) for j, n in enumerate(new)], Hq, tail=4,
                      slots=[s if n else -1 for s, n in zip(b.slot, new)])
    assert np.all(got[-4:] == 7)
    r = 0
    for j, n in enumerate(new):
        if n:
            ref, tol = b.reference(q[r:r + n], j, np.arange(P, P + n))
            assert np.all(np.abs(got[r:r + n] - ref) <= tol), j
        r += n


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_prefill_of_few_rows_among_many_empty_places(dtype):
    """16 rows of five sequences among 2^20 places, as a step of fixed size may
    hold: each place without rows is no work of its own."""
    rng = np.random.default_rng(20)
    P, Hq, Hkv, hd, places = 70, 32, 8, 128, 1 << 20
    at, new, ctx = [0, 5, 64, 70000, places - 1], [1, 6, 1, 3, 5], [130, 76, 71, 73, 200]
    b = Batch(rng, dtype, Hkv, hd, P, ctx)
    q = values(rng, (16, Hq, hd), dtype)
    n, slot, pos = np.zeros(places, int), np.full(places, -1), np.full(places, -1)
    n[at], slot[at], pos[at] = new, b.slot, np.subtract(ctx, new)
    start, qd = i32(np.concatenate([[0], np.cumsum(n)])), torch.from_numpy(q).to(TYPES[dtype]).to(DEV)
    for max_new in (1, 6):                # one row a sequence, and all
        out = torch.full_like(qd, 7.0)
        ws = torch.empty(lp.prefix_prefill_attention_ws_bytes(16, Hq, Hkv, hd, P, 200), dtype=torch.uint8, device=DEV)
        lp.op_prefix_prefill_attention(qd, out, b.kc, b.vc, b.pre_t, P, i32(b.table), start, i32(slot), i32(pos), max_new,
                                       200, ws)
        got, r = out.double().cpu().numpy(), 0
        for j, (x, c) in enumerate(zip(new, ctx)):
            rows = min(x, max_new)
            ref, tol = b.reference(q[r:r + rows], j, np.arange(c - x, c - x + rows))
            assert np.all(np.abs(got[r:r + rows] - ref) <= tol), j
            r += x


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd", [("f16", 8, 2, 128), ("bf16", 2, 2, 64), ("f32", 4, 2, 64)])
def test_infinite_values_inside_a_long_prefix(dtype, Hq, Hkv, hd):
    """Few prompts over a prefix that is split: rows before an infinite value keep their results to the bit."""
    rng = np.random.default_rng(77)
    P, bad = 2000, 930
    b = Batch(rng, dtype, Hkv, hd, P, [P + 30, 960, 5, P + 300])
    seqs = [(0, P, 30), (1, 900, 60), (2, 0, 5), (3, P + 280, 20)]
    q = values(rng, (115, Hq, hd), dtype)
    clean = run_prefill(b, q, seqs, Hq)
    b.vc[int(b.pre[bad // 64]), :, :, bad % 64] = float("inf")
    got = run_prefill(b, q, seqs, Hq)
    r = 0
    for j, p, n in seqs:
        ref, tol = b.reference(q[r:r + n], j, np.arange(p, p + n))
        assert np.all(np.abs(clean[r:r + n] - ref) <= tol)
        for i in range(n):
            if p + i < bad:
                assert np.array_equal(got[r + i], clean[r + i]), (j, i)
            else:
                assert not np.isfinite(got[r + i]).any(), (j, i)
        r += n


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_rows_past_max_new(dtype):
    """Of a sequence with more rows than max_new the first max_new are right,
    and those of the next sequences."""
    rng = np.random.default_rng(8)
    P, Hq, Hkv, hd = 100, 8, 2, 64
    b = Batch(rng, dtype, Hkv, hd, P, [P + 90, P + 20])
    q = values(rng, (112, Hq, hd), dtype)
    got = run_prefill(b, q, [(0, P, 90), (1, P, 20)], Hq, max_new=40, tail=2)
    for j, r, n in ((0, 0, 40), (1, 90, 20)):
        ref, tol = b.reference(q[r:r + n], j, np.arange(P, P + n))
        assert np.all(np.abs(got[r:r + n] - ref) <= tol)
    assert np.all(got[110:] == 7)


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd", [("f16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 64)])
def test_scores_of_minus_infinity(dtype, Hq, Hkv, hd):
    """Infinite keys: rows that they score minus infinity leave them out, get
    zeros where every key is such a one, and NaN where a score is plus infinity."""
    rng = np.random.default_rng(hd + Hq)
    P, ctx = 300, [301, 420, 300, 1200]
    b = Batch(rng, dtype, Hkv, hd, P, ctx)

    def rows_of(n):             # the first dimension's sign decides
        q = values(rng, (n, Hq, hd), dtype)
        q[..., 0] = np.where(np.arange(n) % 4 == 3, 1.0, -1.0)[:, None]
        return q

    def infinite(j, lo, hi):
        for p in range(lo, hi):
            b.kc[int(b.pre[p // 64] if p < P else b.table[b.slot[j], p // 64]), :, p % 64, 0] = float("inf")

    def check(got, q, j, p, gone):
        keep = np.array([i for i in range(p + 1) if not any(lo <= i < hi for k, lo, hi in gone if k in (j, None))], int)
        if (q[0, 0, 0] > 0 and len(keep) <= p):
            assert np.isnan(got).all(), (j, p)
        elif not len(keep):
            assert np.all(got == 0), (j, p)
        else:
            K, V = b.K[j][keep], b.V[j][keep]
            ref, mag = (T.attention(q, K, v, [p], keep, Hkv) for v in (V, np.abs(V)))
            assert np.all(np.abs(got - ref) <= bound(dtype, q, K, V, ref, mag)), (j, p)

    # a few keys in both; then the whole prefix and the first own keys
    gone = [(None, 100, 140), (3, 301, 310), (3, 700, 900)]
    for step in range(2):
        for j, lo, hi in gone:
            infinite(j, lo, hi)
        for n in (4, 44):       # few rows, and a batch that fills a tile
            rows = [(m % 4, [ctx[m % 4] - 1, 130, 99, 299, 311 if m % 4 == 1 else 250][m % 5]) for m in range(n)]
            q = rows_of(n)
            got = run_decode(b, q, rows, Hq)
            for m, (j, p) in enumerate(rows):
                check(got[m:m + 1], q[m:m + 1], j, p, gone)
        seqs = [(1, 290, 130), (2, 90, 60), (3, 1150, 50)]
        q, r = rows_of(240), 0
        got = run_prefill(b, q, seqs, Hq)
        for j, p, n in seqs:
            for i in range(n):
                check(got[r + i:r + i + 1], q[r + i:r + i + 1], j, p + i, gone)
            r += n
        gone = [(None, 0, 300), (3, 300, 310), (3, 700, 900)]


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_sequences_that_leave_the_rows(dtype):
    """Entries of seq_start below 0 and above the rows count as these; a negative seq_pos is no row with keys."""
    rng = np.random.default_rng(4)
    P, Hq, Hkv, hd, n = 100, 4, 2, 64, 50
    b = Batch(rng, dtype, Hkv, hd, P, [P + 60] * 3)
    q = values(rng, (n, Hq, hd), dtype)
    for max_new in (n, 100):
        out = torch.full((n, Hq, hd), 7.0, dtype=TYPES[dtype], device=DEV)
        ws = torch.empty(lp.prefix_prefill_attention_ws_bytes(n, Hq, Hkv, hd, P, P + 60), dtype=torch.uint8, device=DEV)
        lp.op_prefix_prefill_attention(torch.from_numpy(q).to(TYPES[dtype]).to(DEV), out, b.kc, b.vc, b.pre_t, P, i32(b.table),
                                       i32([-9, 12, 30, 70, 90]), i32([b.slot[0], b.slot[1], b.slot[2], b.slot[0]]),
                                       i32([P, -3, P + 20, 5]), max_new, P + 60, ws)
        got = out.double().cpu().numpy()
        for j, r0, r1, p in ((0, 0, 12, P), (2, 30, 50, P + 20)):
            ref, tol = b.reference(q[r0:r1], j, np.arange(p, p + r1 - r0))
            assert np.all(np.abs(got[r0:r1] - ref) <= tol), j
        assert np.all(got[12:30] == 0)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_the_largest_batches_that_always_fit(dtype):
    """Rows times heads times (16 + max_ctx / 4,096) just under 2^22, of which some rows are looked at."""
    rng = np.random.default_rng(22)
    M, Hq, Hkv, hd, P, ctx = 4070, 64, 8, 64, 100, [101, 228, 300]
    assert M * Hq * (16 + 300 / 4096) <= 1 << 22 < (M + 10) * Hq * (16 + 300 / 4096)
    b = Batch(rng, dtype, Hkv, hd, P, ctx)
    q = values(rng, (M, Hq, hd), dtype)
    rows = [(m % 3, ctx[m % 3] - 1) for m in range(M)]
    got = run_decode(b, q, rows, Hq)
    some = [0, 1, 2, 2047, 2048, 3001, M - 2, M - 1]
    for m in some:
        j, p = rows[m]
        ref, tol = b.reference(q[m:m + 1], j, [p])
        assert np.all(np.abs(got[m:m + 1] - ref) <= tol), m
    got = run_prefill(b, q, [(j, p, 1) for j, p in rows], Hq)
    for m in some:
        j, p = rows[m]
        ref, tol = b.reference(q[m:m + 1], j, [p])
        assert np.all(np.abs(got[m:m + 1] - ref) <= tol), m


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_caches_past_4_gib(dtype):
    """Blocks whose byte (f32: also element) offsets pass 32 bits: what a small cache gives, to the bit."""
    rng = np.random.default_rng(21)
    Hq, Hkv, hd, P = 16, 8, 128, 200
    ctx = [P + 1 + 40 * i for i in range(12)]
    b = Batch(rng, dtype, Hkv, hd, P, ctx)
    n = 34000                     # of 131,072 or 262,144 bytes
    big_k = torch.empty(n, Hkv, 64, hd, dtype=TYPES[dtype], device=DEV)
    big_v = torch.empty(n, Hkv, hd, 64, dtype=TYPES[dtype], device=DEV)
    big_k[-b.n_blocks:] = b.kc
    big_v[-b.n_blocks:] = b.vc
    up = n - b.n_blocks

    def call(f, *args):
        small = f(b, *args)
        keep = b.kc, b.vc, b.pre, b.pre_t, b.table
        b.kc, b.vc, b.pre, b.pre_t, b.table = big_k, big_v, b.pre + up, b.pre_t + up, np.where(b.table >= 0, b.table + up, -1)
        large = f(b, *args)
        b.kc, b.vc, b.pre, b.pre_t, b.table = keep
        assert np.isfinite(small).all() and np.array_equal(small, large)

    q = values(rng, (700, Hq, hd), dtype)
    for m in (2, 12):             # few rows, and many
        call(run_decode, q[:m], [(j, ctx[j] - 1) for j in range(m)], Hq)
    rows = [(j, ctx[j] - 1) for j in range(12)] * 12
    call(run_decode, q[:144], rows, Hq)
    call(run_prefill, q[:100], [(0, P, 1), (11, 300, 99)], Hq)
    entry = torch.arange(n * 64 - 70, n * 64 - 5, dtype=torch.int64, device=DEV)
    qkv = torch.randn(65, (Hq + 2 * Hkv) * hd, device=DEV)
    cos, sin = (torch.from_numpy(x).to(DEV) for x in rope_tables(65, hd))
    pos, qo = torch.arange(65, dtype=torch.int32, device=DEV), torch.empty(65, Hq, hd, dtype=TYPES[dtype], device=DEV)
    lp.op_qkv_append(qkv, cos, sin, pos, entry, qo, big_k, big_v)
    small_k, small_v = torch.zeros_like(big_k[:2]), torch.zeros_like(big_v[:2])
    lp.op_qkv_append(qkv, cos, sin, pos, entry - (n - 2) * 64, qo, small_k, small_v)
    for s in (0, 1):
        lo, hi = (58, 64) if s == 0 else (0, 59)
        assert torch.equal(big_k[n - 2 + s][:, lo:hi], small_k[s][:, lo:hi])
        assert torch.equal(big_v[n - 2 + s][:, :, lo:hi], small_v[s][:, :, lo:hi])
        assert small_k[s][:, lo:hi].any()


def counted_prefill(monkeypatch, b, q, seqs, Hq, **how):
    """run_prefill, and the parts that its rows were computed in, from what was
    written of the workspace: rows x heads x parts x (head_dim + 2) fp32 numbers,
    none for one part that goes straight to the output."""
    used, call = [], lp.op_prefix_prefill_attention
    monkeypatch.setattr(lp, "op_prefix_prefill_attention", lambda *args: (used.append(args[-1]), call(*args)))
    got = run_prefill(b, q, seqs, Hq, **how)
    monkeypatch.undo()
    written = (used[0].view(torch.int32) != -1).nonzero()
    return got, (int(written.max()) + 1) / (q.shape[0] * Hq * (b.hd + 2)) if len(written) else 0


@gpu
@pytest.mark.parametrize("dtype,Hq,hd,P", [("f16", 32, 64, 8300), ("bf16", 16, 128, 0)])
def test_one_walk_over_more_than_128_blocks(monkeypatch, dtype, Hq, hd, P):
    """More blocks than a wave holds the places of at a time, three times over:
    prompts in one walk of prefix and own blocks, one inside the prefix, a block
    missing in the middle, and infinite values that the earlier rows' second
    walk has to pass."""
    rng = np.random.default_rng(hd)
    Hkv, first, new = 2, 8300 + 100, 1000
    b = Batch(rng, dtype, Hkv, hd, P, [first + new, 6900])
    q = values(rng, (1100, Hq, hd), dtype)
    gone = 90                                           # an entry of both sequences
    b.table[b.slot[0], gone], b.table[b.slot[1], gone] = -1, -1
    if P:
        b.pre[gone] = -1
        b.pre_t = i32(b.pre)
    seqs = [(0, first, new), (1, 6800, 100)]
    clean, parts = counted_prefill(monkeypatch, b, q, seqs, Hq)
    assert parts == 0 and (first + new) // 64 > 128     # one walk
    r = 0
    for j, p, n in seqs:
        some = np.unique(np.concatenate([np.arange(0, n, 97), [n - 1]]))
        K, V = b.K[j], b.V[j]
        keep = np.setdiff1d(np.arange(len(K)), np.arange(64 * gone, 64 * gone + 64))
        ref, mag = (T.attention(q[r:r + n][some], K[keep], v[keep], p + some, keep, Hkv) for v in (V, np.abs(V)))
        tol = bound(dtype, q[r:r + n][some], K[keep], V[keep], ref, mag)
        assert np.all(np.abs(clean[r:r + n][some] - ref) <= tol), j
        r += n
    # rows before an infinite value keep their results to the bit, others are not finite
    for j, bad, r0, r1 in ((0, first + 517, 517, 1000), (1, 6850, 1050, 1100)):
        blk = int(b.pre[bad // 64] if bad < P else b.table[b.slot[j], bad // 64])
        old = b.vc[blk, :, :, bad % 64].clone()
        b.vc[blk, :, :, bad % 64] = float("inf")
        got, parts = counted_prefill(monkeypatch, b, q, seqs, Hq)
        b.vc[blk, :, :, bad % 64] = old
        behind = np.arange(r0, r1)
        if bad < P:
            behind = np.concatenate([np.arange(1000), behind])      # the other sequence reads it too
        before = np.setdiff1d(np.arange(1100), behind)
        assert parts == 0 and not np.isfinite(got[behind]).any()
        assert np.array_equal(got[before], clean[before])


@gpu
@pytest.mark.parametrize("dtype,Hq,P", [("f16", 8, 100), ("f16", 8, 0), ("f32", 1, 0), ("f32", 1, 100)])
def test_join_of_more_than_64_parts(monkeypatch, dtype, Hq, P):
    """Few new tokens after a long context of their own: the parts after the
    64th, with larger scores than those before; short contexts below the same
    max_ctx, whose later parts are empty; and rows whose first 64 parts are."""
    rng = np.random.default_rng(P + Hq)
    Hkv, hd, top, new = 1, 64, 60000, 30
    b = Batch(rng, dtype, Hkv, hd, P, [top, P + 300])
    b.kc[b.table[b.slot[0], 600:938]] *= 2              # exact
    b.K[0][600 * 64:] *= 2
    q = values(rng, (new, Hq, hd), dtype)

    def check(got, q, j, positions, keep):
        K, V = b.K[j][keep], b.V[j][keep]
        ref, mag = (T.attention(q, K, v, positions, keep, Hkv) for v in (V, np.abs(V)))
        assert np.all(np.abs(got - ref) <= bound(dtype, q, K, V, ref, mag)), j

    got, parts = counted_prefill(monkeypatch, b, q, [(0, top - new, new)], Hq)
    assert parts > 64
    check(got, q, 0, np.arange(top - new, top), np.arange(top))
    got, parts = counted_prefill(monkeypatch, b, q, [(1, P + 270, new)], Hq, max_ctx=top)
    assert parts > 64
    check(got, q, 1, np.arange(P + 270, P + 300), np.arange(P + 300))
    b.table[b.slot[0], :650] = -1
    if P:
        b.pre_t = i32(np.full(len(b.pre), -1))
    got, parts = counted_prefill(monkeypatch, b, q, [(0, top - new, new)], Hq)
    assert parts > 64 and 650 / (938 / parts) > 64 + 4  # the prefix's parts and own ones before the first kept
    check(got, q, 0, np.arange(top - new, top), np.arange(650 * 64, top))


@gpu
def test_graphs_that_share_a_workspace():
    """A prefill and a decode step captured with the same workspace, replayed in
    turn with eager work between, against the eager results."""
    rng = np.random.default_rng(30)
    Hq, Hkv, hd, P, n = 32, 8, 128, 900, 20
    b = Batch(rng, "f16", Hkv, hd, P, [P + 60 + i for i in range(n)])
    table, slot, top, new = i32(b.table), i32(b.slot), P + 100, 30
    qp = torch.from_numpy(values(rng, (n * new, Hq, hd), "f16")).half().to(DEV)
    qd = torch.from_numpy(values(rng, (n, Hq, hd), "f16")).half().to(DEV)
    start, first = i32(np.arange(n + 1) * new), i32([P + 10] * n)
    pos = i32([P + 59 + i for i in range(n)])
    ws = torch.empty(max(lp.prefix_decode_attention_ws_bytes(n, Hq, Hkv, hd, P, top),
                         lp.prefix_prefill_attention_ws_bytes(n * new, Hq, Hkv, hd, P, top)), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(qp), torch.zeros_like(qd)]

    def prefill():
        lp.op_prefix_prefill_attention(qp, outs[0], b.kc, b.vc, b.pre_t, P, table, start, slot, first, new, top, ws)

    def decode():
        lp.op_prefix_decode_attention(qd, outs[1], b.kc, b.vc, b.pre_t, P, table, slot, pos, top, ws)

    want, graphs = [], []
    for k, f in enumerate((prefill, decode)):
        f()
        torch.cuda.synchronize()
        want.append(outs[k].clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            f()
        graphs.append(graph)
    for _ in range(4):
        for k in (0, 1):
            outs[k].fill_(9)
            ws.random_(0, 256)
            graphs[k].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[k], want[k])
            assert torch.isfinite(outs[k]).all()


# ------------------------------------------------------------------ refusals (no GPU is touched)

F16, F32, OK, EINVAL = lp.LP_F16, lp.LP_F32, lp.LP_OK, lp.LP_EINVAL
A = 1 << 20  # an aligned address that is never read: every call below returns before a launch


def test_block_tables_refusals():
    f = lp.lib().lp_op_block_tables
    good = [A, A, A, 2, A, 64, A, 8, A, A, 4, 8, A, A, A, A, A, 10, None]

    def call(**bad):
        names = ("slot", "cached", "lengths", "n", "pre", "P", "free", "n_free", "head", "table", "n_slots", "wide",
                 "seq_start", "free_start", "row_slot", "row_pos", "row_entry", "max_rows", "stream")
        return f(*[bad.get(k, v) for k, v in zip(names, good)])

    assert call(n=0) == OK
    assert f(None, None, None, 0, None, 0, None, 0, None, None, 1, 1, None, None, None, None, None, 0, None) == OK
    for bad in (dict(n=-1), dict(P=-1), dict(P=(1 << 30) + 1), dict(n_free=-1), dict(n_slots=0), dict(wide=0),
                dict(max_rows=-1), dict(n=(1 << 30) + 1)):
        assert call(**bad) == EINVAL, bad
        assert call(n=0, **{k: v for k, v in bad.items() if k != "n"}) == (EINVAL if "n" not in bad else OK)
    for k in ("slot", "cached", "lengths", "pre", "free", "head", "table", "seq_start", "free_start", "row_slot",
              "row_pos", "row_entry"):
        assert call(**{k: None}) == EINVAL, k


def test_qkv_append_refusals():
    f = lp.lib().lp_op_qkv_append
    names = ("dtype", "qkv", "ld", "cos", "sin", "n_pos", "pos", "entry", "rows", "q", "k", "v", "n_blocks", "Hq", "Hkv",
             "hd", "stream")
    good = [F16, A, 1536, A, A, 100, A, A, 3, A, A, A, 5, 8, 2, 128, None]

    def call(**bad):
        return f(*[bad.get(k, v) for k, v in zip(names, good)])

    assert call(rows=0) == OK
    assert call(rows=0, qkv=None, cos=None, sin=None, pos=None, entry=None, q=None, k=None, v=None) == OK
    for bad in (dict(dtype=7), dict(ld=1534), dict(ld=1537), dict(n_pos=0), dict(rows=-1), dict(n_blocks=0), dict(Hq=9),
                dict(Hkv=0), dict(hd=96)):
        assert call(**bad) == EINVAL, bad
        assert call(**{"rows": 0, **bad}) == EINVAL, bad
    for k in ("qkv", "cos", "sin", "pos", "entry", "q", "k", "v"):
        assert call(**{k: None}) == EINVAL, k
    for bad in (dict(qkv=A + 4), dict(cos=A + 4), dict(sin=A + 4), dict(q=A + 8), dict(k=A + 2), dict(v=A + 8)):
        assert call(**bad) == EINVAL, bad


@pytest.mark.parametrize("decode", [True, False])
def test_prefix_attention_refusals(decode):
    L = lp.lib()
    f = L.lp_op_prefix_decode_attention if decode else L.lp_op_prefix_prefill_attention
    size = L.lp_op_prefix_decode_attention_ws_bytes if decode else L.lp_op_prefix_prefill_attention_ws_bytes
    head = dict(dtype=F16, q=A, out=A, k=A, v=A, n_blocks=50, pre=A, P=100, table=A, n_slots=4, wide=8)
    mid = dict(slot=A, pos=A, rows=4) if decode else dict(start=A, slot=A, pos=A, n=2, rows=40, max_new=30)
    tail = dict(Hq=8, Hkv=2, hd=128, max_ctx=500, ws=A, ws_bytes=1 << 40, stream=None)
    good = {**head, **mid, **tail}

    def call(**bad):
        return f(*[bad.get(k, v) for k, v in good.items()])

    pointers = [k for k in ("q", "out", "k", "v", "pre", "table", "start", "slot", "pos", "ws") if k in good]
    assert call(rows=0) == OK and call(**{"rows": 0, **dict.fromkeys(pointers)}) == OK
    if not decode:
        assert call(n=0) == OK and call(n=-1) == EINVAL and call(max_new=0) == EINVAL
    for bad in (dict(dtype=9), dict(rows=-1), dict(P=-1), dict(P=(1 << 30) + 1), dict(n_blocks=0), dict(n_slots=0), dict(wide=0),
                dict(wide=7), dict(Hq=9), dict(Hkv=0), dict(hd=80), dict(max_ctx=0), dict(max_ctx=(1 << 30) + 1),
                dict(rows=1 << 28)):
        assert call(**bad) == EINVAL, bad
        if "rows" not in bad:
            assert call(**{"rows": 0, **bad}) == EINVAL, bad
    for k in pointers:
        assert call(**{k: None}) == EINVAL, k
    for k in ("q", "out", "k", "v", "ws"):
        assert call(**{k: A + 8}) == EINVAL, k
    need = size(good["rows"], 8, 2, 128, 100, 500)
    assert need > 0 and call(ws_bytes=need - 1) == EINVAL
    assert size(-1, 8, 2, 128, 100, 500) == 0 and size(4, 8, 3, 128, 100, 500) == 0 and size(4, 8, 2, 96, 100, 500) == 0
    assert "prefix attention" in L.lp_last_error(None).decode()


def test_binding_refuses_tensors_that_do_not_fit():
    """Wrong devices, types, shapes and layouts raise before the library is called."""
    h = lambda *shape: torch.zeros(*shape, dtype=torch.float16)
    n = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    ws = torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        lp.op_prefix_decode_attention(h(2, 4, 64), h(2, 4, 64), h(3, 2, 64, 64), h(3, 2, 64, 64), n(1), 64, n(2, 3), n(2),
                                      n(2), 70, ws)
    with pytest.raises(ValueError, match="GPU"):
        lp.op_block_tables(n(2), n(2), n(2), n(1), 64, n(4), n(1), n(2, 3), n(3), n(3), n(2), n(2),
                           torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="float"):
        lp.op_qkv_append(torch.zeros(2, 512), torch.zeros(9, 32), torch.zeros(9, 32), n(2), torch.zeros(2, dtype=torch.int64),
                         n(2, 4, 64), n(3, 2, 64, 64), n(3, 2, 64, 64))


@gpu
def test_binding_refuses_shapes_on_the_gpu():
    h = lambda *shape: torch.zeros(*shape, dtype=torch.float16, device=DEV)
    n = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=DEV)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    good = dict(q=h(2, 4, 64), out=h(2, 4, 64), kc=h(3, 2, 64, 64), vc=h(3, 2, 64, 64), prefix_blocks=n(1), prefix_len=64,
                block_table=n(2, 3), row_slot=n(2), row_pos=n(2), max_ctx=70, ws=ws)
    lp.op_prefix_decode_attention(**good)
    for bad in (dict(q=h(2, 4, 128)[:, :, ::2]), dict(out=h(3, 4, 64)), dict(vc=h(3, 2, 64, 32)), dict(prefix_len=65),
                dict(row_slot=n(3)), dict(row_pos=n(2).long()), dict(kc=h(3, 2, 64, 64).float()), dict(block_table=n(3, 2).T),
                dict(row_slot=n(2).cpu())):
        with pytest.raises(ValueError):
            lp.op_prefix_decode_attention(**{**good, **bad})
    with pytest.raises(lp.LPError):
        lp.op_prefix_decode_attention(**{**good, "ws": ws[:64]})
    torch.cuda.synchronize()


@pytest.mark.parametrize("decode", [True, False])
def test_work_past_one_launch_is_refused(decode):
    """Sizes within the limits each, whose workgroups together are too many."""
    L = lp.lib()
    f = L.lp_op_prefix_decode_attention if decode else L.lp_op_prefix_prefill_attention
    for dtype, rows, Hq, Hkv, P, ctx in ((F16, 1 << 22, 8, 2, 100, 500), (F32, 1 << 20, 16, 16, 1 << 20, (1 << 20) + 70),
                                         (F16, 1 << 20, 16, 16, 64, 1 << 29), (F32, 1 << 22, 8, 2, 0, 500)):
        if dtype == F16 and rows == 1 << 20 and not decode:
            continue                      # one workgroup takes all blocks of a tile there
        seqs = [A, A, rows] if decode else [A, A, A, rows, rows, 1]
        args = [dtype, A, A, A, A, 50, A, P, A, 4, 1 << 24, *seqs, Hq, Hkv, 64, ctx, A, 1 << 60, None]
        assert f(*args) == EINVAL, (dtype, rows)
        assert "launch" in L.lp_last_error(None).decode()


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("dtype", [F16, lp.LP_BF16, F32])
def test_row_and_head_pairs_past_one_launch_are_refused(decode, dtype):
    """From 2^25 pairs on, whatever the contexts; the workspace's size, which
    depends on neither dtype nor sequences, is that of the limits alone."""
    L = lp.lib()
    f = L.lp_op_prefix_decode_attention if decode else L.lp_op_prefix_prefill_attention
    size = L.lp_op_prefix_decode_attention_ws_bytes if decode else L.lp_op_prefix_prefill_attention_ws_bytes
    for rows, Hq, Hkv, P, ctx in ((1 << 20, 32, 8, 0, 1), (1 << 20, 32, 8, 64, 50), (1 << 22, 8, 8, 5000, 5100), (1 << 29, 1, 1, 64, 70)):
        seqs = [A, A, rows] if decode else [A, A, A, 1, rows, rows]
        assert f(dtype, A, A, A, A, 50, A, P, A, 4, 1000, *seqs, Hq, Hkv, 64, ctx, A, 1 << 60, None) == EINVAL, (rows, Hq)
        assert "launch" in L.lp_last_error(None).decode()
        assert size(rows, Hq, Hkv, 64, P, ctx) > 0
    assert size((1 << 25) + 1, 32, 8, 64, 64, 70) == size(1, 8, 8, 64, 0, (1 << 30) + 1) == size(1, 8, 8, 64, (1 << 30) + 1, 9) == 0


def test_loads_into_lds_keep_their_wait_states(tmp_path):
    """What is checked of the other kernels' loads into LDS, for these."""
    device_code.test_loads_into_lds_keep_their_wait_states("prefix", tmp_path)
