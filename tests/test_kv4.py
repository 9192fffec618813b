"""A K/V cache held in 4 bits (include/lp_ops.h, last section): quantising as it
is written, reading back, and decode and prefill attention over it, against plain
float64 implementations.  Every place that no row may read holds random bytes, NaN
scales among them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import transformer as T
from paper_2410_02425_amd import lp

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step at 1
gpu = pytest.mark.gpu
MAGS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def ceil64(n):
    return -(-n // 64)


def i32(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


def i64(a):
    return torch.tensor(np.asarray(a, dtype=np.int64), device=DEV)


# ------------------------------------------------------------------ the format, from its definition

def scales(amax):
    """Scale of groups from their largest magnitudes (float64): found by trying the grid's steps."""
    amax = np.asarray(amax, dtype=np.float64)
    t = np.where(np.isfinite(amax), amax, 0.0) / 6.0
    with np.errstate(divide="ignore"):
        e = np.maximum(np.floor(np.log2(t)) - 5, -23)
    step = np.exp2(e)
    m = np.floor(t / step) - 1  # below, in case the logarithm or division rounded up
    for _ in range(3):
        m = np.where(6.0 * m * step < amax, m + 1, m)
    s = np.minimum(np.maximum(m, 0) * step, 10752.0)
    return np.where(np.isfinite(amax), s, np.nan)


def quantise(x):
    """Codes (0 .. 15) and scales of x [..., hd], groups of 32."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    with np.errstate(invalid="ignore"):
        amax = np.abs(g).max(-1)
    amax = np.where(np.isfinite(g).all(-1), amax, np.inf)
    s = scales(amax)
    order = [0, 2, 4, 6, 1, 3, 5, 7]  # even codes first: they win ties
    with np.errstate(invalid="ignore"):
        a = np.minimum(np.abs(g), 6 * s[..., None])  # past 6 s, 6 is the nearest (and no difference is lost)
        err = np.abs(a[..., None] - MAGS[order] * s[..., None, None])
    code = np.where(np.isfinite(s)[..., None], np.asarray(order)[np.argmin(np.nan_to_num(err), -1)], 0)
    code = np.where(s[..., None] == 0, 0, code)
    return (code + 8 * np.signbit(g)).reshape(x.shape).astype(np.uint8), s


def held(code, s):
    """The values that codes [..., hd] and scales [..., hd / 32] stand for."""
    v = np.where(code >= 8, -1.0, 1.0) * MAGS[code & 7]
    return (v.reshape(*code.shape[:-1], code.shape[-1] // 32, 32) * s[..., None]).reshape(code.shape)


def byte_tables(hd):
    """(byte, half) of every (position, dim) of K and V, and of the scales of every (position, group)."""
    J = hd // 32
    p, d = np.meshgrid(np.arange(64), np.arange(hd), indexing="ij")
    j, o = d // 32, d % 32
    k = p * (hd // 2) + 4 * J * (o // 8) + 4 * j + o % 8 // 2
    y = J * (o // 2) + j
    v = 36 * hd + ((p // 4 * (hd // 8) + y // 4) * 4 + p % 4) * 4 + y % 4
    p, g = np.meshgrid(np.arange(64), np.arange(J), indexing="ij")
    return k, v, d % 2, 32 * hd + (p * J + g) * 2, 68 * hd + (g * 64 + p) * 2


def put(block, p, k, v):
    """Stores K and V rows (codes, scales) at place p of a block's bytes [Hkv, 72 hd]."""
    hd = k[0].shape[-1]
    kb, vb, half, ks, vs = byte_tables(hd)
    for (code, s), at, sat in ((k, kb, ks), (v, vb, vs)):
        for x in (0, 1):
            b = at[p][half[p] == x]
            keep = block[:, b] & (0xF0 if x == 0 else 0x0F)
            block[:, b] = keep | (code[:, half[p] == x] << (4 * x))
        raw = s.astype(np.float16).view(np.uint16)
        block[:, sat[p]] = raw & 255
        block[:, sat[p] + 1] = raw >> 8


def get(block, p):
    """K and V values of place p of a block's bytes [Hkv, 72 hd]."""
    hd = block.shape[1] // 72
    kb, vb, half, ks, vs = byte_tables(hd)
    out = []
    for at, sat in ((kb, ks), (vb, vs)):
        code = block[:, at[p]] >> (4 * half[p]) & 15
        s = (block[:, sat[p]].astype(np.uint16) | block[:, sat[p] + 1].astype(np.uint16) << 8).view(np.float16)
        out.append(held(code, s.astype(np.float64)))
    return out


def noise(rng, n_blocks, Hkv, hd):
    """A cache of random bytes, a fourth of its scales NaN or infinite."""
    c = rng.integers(0, 256, (n_blocks, Hkv, 72 * hd), dtype=np.uint8)
    for lo in (32 * hd, 68 * hd):
        part = c[:, :, lo:lo + 4 * hd].copy().view(np.uint16)
        odd = rng.random(part.shape) < 0.25
        part[odd] = rng.choice(np.array([0x7E00, 0x7C00, 0xFE01, 0xFC00], dtype=np.uint16), odd.sum())
        c[:, :, lo:lo + 4 * hd] = part.view(np.uint8)
    return c


def test_the_reference_format():
    """What tests build on: bytes are used once each, and values come back as the nearest of the grid."""
    for hd in (64, 128):
        kb, vb, half, ks, vs = byte_tables(hd)
        used = np.concatenate([(kb * 2 + half).ravel(), (vb * 2 + half).ravel()]
                              + [(x.ravel() * 2)[:, None] + np.arange(4) for x in (ks, vs)], axis=None)
        assert np.array_equal(np.sort(used), np.arange(144 * hd))
        rng = np.random.default_rng(hd)
        x = rng.standard_normal((2, 64, 3, hd))
        block = noise(rng, 1, 3, hd)[0]
        for p in range(64):
            put(block, p, quantise(x[0, p]), quantise(x[1, p]))
        for p in range(64):
            for got, want in zip(get(block, p), x[:, p]):
                assert np.all(np.abs(got - want) <= np.abs(want).max() / 6 * (1 + 2.0 ** -5))
    assert scales([0.0, 6.0, 6.0 + 1e-9, 6 * 2.0 ** -23, 1e-30, 64512.0, 7e4, np.inf, np.nan]).tolist()[:7] == \
        [0.0, 1.0, 1 + 2.0 ** -5, 2.0 ** -23, 2.0 ** -23, 10752.0, 10752.0]
    x = np.zeros((1, 32))
    x[0, :9] = [6.0, 0.25, 0.75, 1.25, 1.75, -2.5, 3.5, 5.0, 0.2500001]
    assert quantise(x)[0][0, :9].tolist() == [7, 0, 2, 2, 4, 12, 6, 6, 1]


# ------------------------------------------------------------------ append

def rope_tables(n_pos, hd):
    c, s = T.rope_cos_sin(np.arange(n_pos), hd, 10000.0)
    return c.astype(np.float32), s.astype(np.float32)


def run_append(dtype, x, width, cos, sin, pos, entry, Hq, hd, cache):
    q = torch.full((len(pos), Hq, hd), 7.0, dtype=TYPES[dtype], device=DEV)
    cd = torch.from_numpy(cache.copy()).to(DEV)
    lp.op_kv4_append(torch.from_numpy(x).to(DEV)[:, :width], torch.from_numpy(cos).to(DEV),
                     torch.from_numpy(sin).to(DEV), i32(pos), i64(entry), q, cd)
    torch.cuda.synchronize()
    return q.double().cpu().numpy(), cd.cpu().numpy()


APPEND_CASES = [
    # dtype, Hq, Hkv, hd, positions of each run of rows, columns past the projection's
    ("f16", 32, 8, 128, [(0, 1)], 0), ("bf16", 32, 8, 128, [(5, 1)] * 3 + [(63, 1), (64, 1)], 0),
    ("f16", 8, 2, 64, [(0, 200), (61, 9)], 0), ("bf16", 6, 2, 128, [(3, 130), (250, 70)], 6),
    ("f32", 4, 4, 64, [(0, 37), (64, 64)], 0), ("f32", 5, 1, 128, [(1, 63), (127, 2)], 2),
    ("f16", 40, 40, 128, [(30, 70)], 2), ("f16", 3, 3, 64, [(7, 8), (0, 8), (56, 16)], 0),
]


def append_rows(rng, runs, extra_entries=True):
    """Positions and entries of runs of rows in blocks of their own, and between them rows that have no position, a
    position past the tables or no entry."""
    n_pos = max(p + n for p, n in runs)
    n_blocks = sum(ceil64(p + n) for p, n in runs) + 2
    blocks = rng.permutation(n_blocks)[: n_blocks - 2]
    pos, entry, at = [], [], 0
    for p, n in runs:
        k = np.arange(p, p + n)
        pos += k.tolist() + [-1, n_pos, p]
        entry += (blocks[at + k // 64] * 64 + k % 64).tolist() + [5, 9, [-1, n_blocks * 64, 2 ** 40][at % 3]]
        at += ceil64(p + n)
    return n_pos, n_blocks, pos, entry


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,runs,extra", APPEND_CASES)
def test_append_of_unrotated_rows_is_exact(dtype, Hq, Hkv, hd, runs, extra):
    """With every angle 0 the rotation changes nothing, and each byte is defined:
    codes and scales of the rows that have an entry, the others as they were."""
    rng = np.random.default_rng(Hq * 7 + len(runs))
    n_pos, n_blocks, pos, entry = append_rows(rng, runs)
    rows, width = len(pos), (Hq + 2 * Hkv) * hd
    x = rng.standard_normal((rows, width + extra)).astype(np.float32)
    # groups whose values lie on the grid and on its borders, of one size, zero, past the range, and not finite
    g = x[:, :width].reshape(rows, -1, 32)
    kind = rng.integers(0, 12, g.shape[:2])
    g[kind == 0] = (rng.choice([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6], g.shape)
                    * rng.choice([-1, 1], g.shape) * np.exp2(rng.integers(-20, 10, (rows, g.shape[1], 1))))[kind == 0]
    g[kind == 1] *= np.exp2(rng.integers(-40, 17, g.shape))[kind == 1]
    g[kind == 2] = 0
    g[kind == 3, 5] = rng.choice([np.inf, -np.inf, np.nan, 7e4, -3e38, 64512, 1e-42], (kind == 3).sum())
    cos, sin = np.ones((n_pos, hd // 2), np.float32), np.zeros((n_pos, hd // 2), np.float32)
    before = noise(rng, n_blocks, Hkv, hd)
    q, cache = run_append(dtype, x, width, cos, sin, pos, entry, Hq, hd, before)
    want = before.copy()
    h = x[:, :width].reshape(rows, Hq + 2 * Hkv, hd)
    # x cos - y sin: 0 times an infinity or NaN is NaN, in the partner dim's group too
    with np.errstate(invalid="ignore"):
        a, b = h[:, :Hq + Hkv, :hd // 2], h[:, :Hq + Hkv, hd // 2:]
        rot = np.concatenate([a - b * np.float32(0), b + a * np.float32(0)], axis=2)
    live = [r for r, (p, e) in enumerate(zip(pos, entry)) if 0 <= p < n_pos and 0 <= e < n_blocks * 64]
    for r in live:
        put(want[entry[r] // 64], entry[r] % 64, quantise(rot[r, Hq:]), quantise(h[r, Hq + Hkv:]))
    # a group with an infinity or NaN reads as NaN whatever its codes; signs of zeros are not defined
    assert np.array_equal(canonical(cache), canonical(want))
    wq = torch.from_numpy(rot[:, :Hq]).to(TYPES[dtype]).double().numpy()
    inside = np.array([0 <= p < n_pos for p in pos])
    assert np.array_equal(q[inside], wq[inside], equal_nan=True) and np.all(q[~inside] == 7)


def canonical(cache):
    """Cache bytes with every NaN scale the same, and codes of NaN groups, and signs of zero codes, cleared."""
    n, Hkv, size = cache.shape
    hd = size // 72
    kb, vb, half, ks, vs = byte_tables(hd)
    out = []
    for at, sat in ((kb, ks), (vb, vs)):
        code = cache[:, :, at] >> (4 * half).astype(np.uint8) & 15
        s = cache[:, :, sat].astype(np.uint16) | cache[:, :, sat + 1].astype(np.uint16) << 8
        bad = np.isnan(s.view(np.float16))
        code = np.where(np.repeat(bad, 32, axis=-1) | (code & 7 == 0), 0, code)
        out += [code.ravel(), np.where(bad, 0x7E00, s).ravel()]
    return np.concatenate(out)


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,runs,extra", APPEND_CASES)
def test_append_rotates(dtype, Hq, Hkv, hd, runs, extra):
    """The rotation is one rounded product and one fused step in fp32 (2^-24 of
    the terms each): q is that rounded to dtype; K's scale is one that a largest
    magnitude within that error has, its values are as near as the nearest, but
    for that error."""
    rng = np.random.default_rng(Hq * 9 + len(runs))
    n_pos, n_blocks, pos, entry = append_rows(rng, runs)
    rows, width = len(pos), (Hq + 2 * Hkv) * hd
    x = rng.standard_normal((rows, width + extra)).astype(np.float32)
    cos, sin = rope_tables(n_pos, hd)
    before = noise(rng, n_blocks, Hkv, hd)
    q, cache = run_append(dtype, x, width, cos, sin, pos, entry, Hq, hd, before)
    h = x[:, :width].astype(np.float64).reshape(rows, Hq + 2 * Hkv, hd)
    u, live = UNIT[dtype], np.zeros((n_blocks, 64), bool)
    for r, (p, e) in enumerate(zip(pos, entry)):
        if not 0 <= p < n_pos:
            assert np.all(q[r] == 7)
            continue
        c, s = cos[p].astype(np.float64), sin[p].astype(np.float64)
        a, b = h[r, :Hq + Hkv, :hd // 2], h[r, :Hq + Hkv, hd // 2:]
        y = np.concatenate([a * c - b * s, b * c + a * s], axis=1)
        off = 2.0 ** -23 * np.concatenate([abs(a * c) + abs(b * s), abs(b * c) + abs(a * s)], axis=1)
        tol = (u if dtype != "f32" else 0) * np.abs(y[:Hq]) * (1 + 2 ** -10) + off[:Hq] + 2.0 ** -25
        assert np.all(np.abs(q[r] - y[:Hq]) <= tol)
        if not 0 <= e < n_blocks * 64:
            continue
        live[e // 64, e % 64] = True
        k, v = get(cache[e // 64], e % 64)
        assert np.array_equal(v, held(*quantise(x[r, :width].reshape(-1, hd)[Hq + Hkv:])))
        y, off = y[Hq:].reshape(Hkv, -1, 32), off[Hq:].reshape(Hkv, -1, 32)
        top = np.abs(y).max(-1)
        sc = cache[e // 64][:, byte_tables(hd)[3][e % 64] + np.array([[0], [1]])].astype(np.uint16)
        sc = (sc[:, 0] | sc[:, 1] << 8).view(np.float16).astype(np.float64)
        assert np.all((scales(top - off.max(-1)) <= sc) & (sc <= scales(top + off.max(-1))))
        near = np.abs(np.abs(y)[..., None] - MAGS * sc[..., None, None]).min(-1)
        assert np.all(np.abs(k.reshape(y.shape) - y) <= near + 2 * off)
    kb, vb, half, ks, vs = byte_tables(hd)
    for blk in range(n_blocks):
        for p in np.flatnonzero(~live[blk]):
            for at in (kb[p], vb[p], ks[p], ks[p] + 1, vs[p], vs[p] + 1):
                assert np.array_equal(cache[blk][:, at], before[blk][:, at])


# ------------------------------------------------------------------ read

@gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("Hkv,hd,rows", [(8, 128, 1), (2, 64, 5), (3, 128, 64), (1, 64, 200), (5, 128, 333), (40, 64, 130)])
@pytest.mark.parametrize("ordered", [True, False])
def test_read(dtype, Hkv, hd, rows, ordered):
    """Every value comes back exactly; rows without an entry on either side, and
    the places that no row names, stay as they were."""
    rng = np.random.default_rng(rows * 3 + hd)
    n_blocks, n_dst = ceil64(rows) + 3, ceil64(rows) + 2
    cache = noise(rng, n_blocks, Hkv, hd)
    # scales of the format: at most 6 significant bits, multiples of 2^-23, up to 10752, and NaN
    for lo in (32 * hd, 68 * hd):
        shape = (n_blocks, Hkv, 2 * hd)
        s = np.minimum(scales(np.abs(rng.standard_normal(shape)) * np.exp2(rng.integers(-30, 17, shape))), 10752.0)
        s[rng.random(shape) < 0.02] = np.nan
        cache[:, :, lo:lo + 4 * hd] = s.astype(np.float16).view(np.uint8)
    if ordered:
        src = np.arange(rows) + 64 + (0 if rows % 64 == 0 else 3)
        dst = np.arange(rows) + (64 if rows % 64 == 0 else 7)
    else:
        src, dst = rng.permutation(n_blocks * 64)[:rows], rng.permutation(n_dst * 64)[:rows]
    if rows > 4:
        src[1], dst[2], src[3] = -1, -1, n_blocks * 64
        dst[4] = n_dst * 64
    kc = torch.full((n_dst, Hkv, 64, hd), 7.0, dtype=TYPES[dtype], device=DEV)
    vc = torch.full((n_dst, Hkv, hd, 64), 7.0, dtype=TYPES[dtype], device=DEV)
    lp.op_kv4_read(torch.from_numpy(cache).to(DEV), i64(src), i64(dst), kc, vc)
    torch.cuda.synchronize()
    wk, wv = np.full(kc.shape, 7.0), np.full(vc.shape, 7.0)
    for s, d in zip(src, dst):
        if 0 <= s < n_blocks * 64 and 0 <= d < n_dst * 64:
            wk[d // 64, :, d % 64], wv[d // 64, :, :, d % 64] = get(cache[s // 64], s % 64)
    assert np.array_equal(kc.double().cpu().numpy(), wk, equal_nan=True)
    assert np.array_equal(vc.double().cpu().numpy(), wv, equal_nan=True)


# ------------------------------------------------------------------ attention

class Batch:
    """Sequences (their context lengths): K and V values per sequence on the
    host, a cache of noise wherever no sequence has an entry, table rows in
    shuffled slots."""

    def __init__(self, rng, dtype, Hkv, hd, ctx, spare_slots=2, scale=1.0, vscale=1.0):
        need = [ceil64(c) for c in ctx]
        n_slots = len(ctx) + spare_slots
        self.n_blocks = sum(need) + 3
        perm = rng.permutation(self.n_blocks)
        self.Hkv, self.hd, self.dtype, self.ctx = Hkv, hd, dtype, ctx
        self.table = np.full((n_slots, max(need + [1]) + 1), -1)
        self.slot = rng.permutation(n_slots)[:len(ctx)]
        self.bytes = noise(rng, self.n_blocks, Hkv, hd)
        at, self.K, self.V = 0, [], []
        for s, c, n in zip(self.slot, ctx, need):
            self.table[s, :n] = perm[at:at + n]
            at += n
            kq, vq = (quantise(rng.standard_normal((c, Hkv, hd)) * f) for f in (scale, vscale))
            for p in range(c):
                self.store(s, p, [x[p] for x in kq], [x[p] for x in vq])
            self.K.append(held(*kq))
            self.V.append(held(*vq))

    def store(self, slot, p, k, v):
        put(self.bytes[self.table[slot, p // 64]], p % 64, k, v)

    def cache(self):
        return torch.from_numpy(self.bytes).to(DEV)

    def reference(self, q, j, positions):
        """Attention of rows q of sequence j at these positions, and its error bound."""
        K, V = self.K[j], self.V[j]
        n = max(positions) + 1
        ref = T.attention(q, K[:n], V[:n], positions, np.arange(n), self.Hkv)
        mag = T.attention(q, K[:n], np.abs(V[:n]), positions, np.arange(n), self.Hkv)
        return ref, bound(self.dtype, q, K[:n], V[:n], ref, mag)


def bound(dtype, q, K, V, ref, mag):
    """Error of softmax(q K^T / sqrt(hd)) V with fp32 scores and sums: a score
    of hd products in hd / 32 groups with a scale each is off by (hd + 12) 2^-24
    of its terms' sizes, which moves numerator and denominator; exp, the sums
    over n keys, the products with V's scales and the joins of parts add (n + 96)
    2^-24.  16-bit kernels round each weight, or weight times V's scale, to fp16
    (2^-11, and at least 2^-25 of the largest: n times that, of values up to
    twice the largest V) and the result (u)."""
    n, Hkv, hd = K.shape
    terms = np.linalg.norm(q, axis=-1).max() * np.linalg.norm(K, axis=-1).max() / np.sqrt(hd)
    tol = (2 * (hd + 12) * 2.0 ** -24 * terms + (n + 96) * 2.0 ** -24) * mag
    if dtype == "f32":
        return tol + 2.0 ** -24 * np.abs(ref)
    small = n * 2.0 ** -24 * np.abs(V).max()
    return tol + (2.0 ** -11 * mag + UNIT[dtype] * np.abs(ref)) * (1 + 2.0 ** -6) + small + 2.0 ** -25


def values(rng, shape, dtype, scale=1.0):
    """Random values that dtype holds exactly, as float64."""
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(TYPES[dtype]).double().numpy()


def run_decode(b, q, rows, Hq, max_ctx=None, slots=None):
    """rows: (sequence, position) of each row; position -1: none."""
    M = len(rows)
    slot = i32([b.slot[j] for j, _ in rows]) if slots is None else i32(slots)
    pos = i32([p for _, p in rows])
    max_ctx = max_ctx or max([p for _, p in rows] + [0]) + 1
    out = torch.full((M, Hq, b.hd), float("nan"), dtype=TYPES[b.dtype], device=DEV)
    qd = torch.from_numpy(q).to(TYPES[b.dtype]).to(DEV)
    need = lp.kv4_decode_attention_ws_bytes(M, Hq, b.Hkv, b.hd, max_ctx)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    lp.op_kv4_decode_attention(qd, out, b.cache(), i32(b.table), slot, pos, max_ctx, ws[:need])
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all()
    return out.double().cpu().numpy()


DECODE_CASES = [
    # dtype, Hq, Hkv, hd, contexts (0: an empty row)
    ("f16", 4, 1, 128, [613]), ("bf16", 32, 8, 128, [65, 64, 63, 1, 0, 130]),
    ("f16", 32, 8, 128, [500 + 37 * i for i in range(20)]), ("f16", 8, 8, 128, [101, 100, 99, 400, 128, 129]),
    ("bf16", 40, 40, 128, [66, 200, 65, 800]), ("f16", 64, 8, 128, [9 * i for i in range(70)]),
    ("f16", 8, 8, 64, [1, 64, 65, 0, 300]), ("bf16", 6, 2, 64, [1, 2, 64, 65]), ("f16", 5, 1, 128, [201, 260, 7]),
    ("bf16", 16, 1, 64, [321] * 9), ("f16", 24, 1, 128, [192, 700]), ("f32", 4, 4, 64, [101, 130, 90, 0, 300]),
    ("f32", 8, 2, 128, [64, 65, 500]), ("f32", 3, 1, 64, [1, 77]), ("f32", 40, 8, 128, [201 + i for i in range(30)]),
    ("bf16", 8, 2, 128, [5001, 3300, 4000]), ("f16", 32, 8, 128, [65 + i for i in range(130)]),
    ("f16", 8, 2, 64, [16, 17, 31, 32, 33, 47, 48, 49, 4097]), ("f32", 17, 1, 128, [16, 33, 1000]),
]


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,ctx", DECODE_CASES)
def test_decode_attention(dtype, Hq, Hkv, hd, ctx):
    rng = np.random.default_rng(ctx[0] * 31 + len(ctx) + Hq)
    b = Batch(rng, dtype, Hkv, hd, ctx)
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
    need = lp.kv4_prefill_attention_ws_bytes(rows, Hq, b.Hkv, b.hd, max_ctx)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    slot = i32([b.slot[j] for j, _, _ in seqs]) if slots is None else i32(slots)
    lp.op_kv4_prefill_attention(qd, out, b.cache(), i32(b.table), seq_start, slot, i32([p for _, p, _ in seqs]),
                                max_new, max_ctx, ws[:need])
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all()
    return out.double().cpu().numpy()


def check_prefill(b, q, got, seqs, start=0):
    at = start
    for j, p, n in seqs:
        if n:
            ref, tol = b.reference(q[at:at + n], j, list(range(p, p + n)))
            err = np.abs(got[at:at + n] - ref)
            assert np.all(err <= tol), (j, p, n, np.nanmax(err / tol))
        at += n


PREFILL_CASES = [
    # dtype, Hq, Hkv, hd, sequences (first position, rows)
    ("f16", 32, 8, 128, [(0, 1)]), ("bf16", 32, 8, 128, [(0, 40), (100, 3), (64, 64), (5, 0), (63, 2)]),
    ("f16", 4, 1, 128, [(0, 547)]), ("bf16", 8, 8, 128, [(300, 130), (0, 129), (1, 17)]),
    ("f16", 8, 2, 64, [(0, 300), (77, 100)]), ("bf16", 6, 2, 64, [(7, 9), (0, 33), (1000, 65)]),
    ("f16", 64, 8, 128, [(200, 50), (0, 20)]), ("f32", 4, 4, 64, [(64, 20), (0, 20), (31, 33)]),
    ("f32", 8, 2, 128, [(0, 100), (450, 7)]), ("f32", 3, 1, 64, [(0, 1), (62, 5)]),
    ("f16", 5, 1, 64, [(128, 64), (0, 64), (64, 1)]), ("bf16", 40, 40, 128, [(15, 49), (1600, 4)]),
    ("f16", 32, 8, 128, [(50 * i, 10 + i) for i in range(12)]), ("bf16", 17, 1, 128, [(400, 90)]),
    ("f16", 16, 2, 128, [(2000, 30)]), ("bf16", 16, 16, 64, [(0, 260), (260, 260)]),
]


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,seqs", PREFILL_CASES)
def test_prefill_attention(dtype, Hq, Hkv, hd, seqs):
    rng = np.random.default_rng(len(seqs) * 31 + Hq + seqs[0][1])
    b = Batch(rng, dtype, Hkv, hd, [p + n for p, n in seqs])
    seqs = [(j, p, n) for j, (p, n) in enumerate(seqs)]
    start, tail = 3, 5
    q = values(rng, (start + sum(n for _, _, n in seqs) + tail, Hq, hd), dtype)
    got = run_prefill(b, q, seqs, Hq, start=start, tail=tail)
    check_prefill(b, q, got, seqs, start)
    assert np.all(got[:start] == 7) and np.all(got[len(got) - tail:] == 7)


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd", [("f16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 64)])
def test_a_service_from_projection_to_read_back(dtype, Hq, Hkv, hd):
    """Tables from lengths, append, prefill, then decode steps, and the contexts
    read back into an ordinary cache over which ordinary decode attention gives
    what the 4-bit one does."""
    rng = np.random.default_rng(hd + Hq)
    n, steps = 3, 3
    lengths = np.array([70, 5, 129])
    total = [ceil64(int(x) + steps) for x in lengths]
    n_blocks, wide = sum(total) + 4, max(total) + 1
    cos, sin = rope_tables(256, hd)
    cd, sd = torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV)
    cache = torch.from_numpy(noise(rng, n_blocks, Hkv, hd)).to(DEV)
    free, head = i32(rng.permutation(n_blocks)), i32([0])
    table, slot = i32(np.full((n + 1, wide), -1)), i32([2, 0, 3])
    cached = np.zeros(n, int)
    K, V = ([np.zeros((0, Hkv, hd)) for _ in range(n)] for _ in range(2))
    tdt, width = TYPES[dtype], (Hq + 2 * Hkv) * hd
    b = Batch.__new__(Batch)
    b.Hkv, b.hd, b.dtype = Hkv, hd, dtype
    for step in range(steps + 1):
        now = lengths + step
        new = now - cached
        rows = int(new.sum())
        start, taken = i32([0] * (n + 1)), i32([0] * (n + 1))
        rslot, rpos, entry = i32([0] * rows), i32([0] * rows), i64([0] * rows)
        lp.op_block_tables(slot, i32(cached), i32(now), None, 0, free, head, table, start, taken, rslot, rpos, entry)
        x = rng.standard_normal((rows, width)).astype(np.float32)
        q = torch.empty(rows, Hq, hd, dtype=tdt, device=DEV)
        out = torch.empty_like(q)
        lp.op_kv4_append(torch.from_numpy(x).to(DEV), cd, sd, rpos, entry, q, cache)
        top = int(now.max())
        if step == 0:
            ws = torch.empty(max(16, lp.kv4_prefill_attention_ws_bytes(rows, Hq, Hkv, hd, top)), dtype=torch.uint8,
                             device=DEV)
            lp.op_kv4_prefill_attention(q, out, cache, table, start, slot, i32(cached), int(new.max()), top, ws)
        else:
            ws = torch.empty(max(16, lp.kv4_decode_attention_ws_bytes(rows, Hq, Hkv, hd, top)), dtype=torch.uint8,
                             device=DEV)
            lp.op_kv4_decode_attention(q, out, cache, table, rslot, rpos, top, ws)
        torch.cuda.synchronize()
        # what the cache now holds is what attention has to read
        bytes_, e, at = cache.cpu().numpy(), entry.tolist(), 0
        for j in range(n):
            for r in range(at, at + int(new[j])):
                k, v = get(bytes_[e[r] // 64], e[r] % 64)
                K[j], V[j] = np.concatenate([K[j], k[None]]), np.concatenate([V[j], v[None]])
                assert np.array_equal(v, held(*quantise(x[r].reshape(-1, hd)[Hq + Hkv:])))
            at += int(new[j])
        b.K, b.V = K, V
        check_prefill(b, q.double().cpu().numpy(), out.double().cpu().numpy(),
                      [(j, int(cached[j]), int(new[j])) for j in range(n)])
        head, cached = taken[n:].clone(), now
    # back into an ordinary cache of the same blocks
    kc = torch.zeros(n_blocks, Hkv, 64, hd, dtype=tdt, device=DEV)
    vc = torch.zeros(n_blocks, Hkv, hd, 64, dtype=tdt, device=DEV)
    host = table.cpu().numpy()
    every = np.concatenate([host[s][np.arange(c) // 64] * 64 + np.arange(c) % 64
                            for s, c in zip([2, 0, 3], cached)])
    lp.op_kv4_read(cache, i64(every), i64(every), kc, vc)
    again = torch.empty_like(out)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    lp.op_decode_attention(q, again, kc, vc, table, rslot, rpos, Hkv, wide * 64, ws)
    torch.cuda.synchronize()
    for j in range(n):
        qj = q[j:j + 1].double().cpu().numpy()
        ref, tol = b.reference(qj, j, [int(cached[j]) - 1])
        tol16 = tol + 2 * UNIT[dtype] * np.abs(V[j]).max() if dtype != "f32" else tol
        assert np.all(np.abs(again[j:j + 1].double().cpu().numpy() - ref) <= tol16)
