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


@gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_append_of_the_least_magnitudes(hd):
    """Groups whose largest magnitude is 0 to 9 times the least of fp32, 2^-149: all but 0 have the
    least scale, 2^-23, also where a sixth of the magnitude is nothing in fp32."""
    rng = np.random.default_rng(149)
    Hq, Hkv, rows = 2, 2, 70
    x = rng.integers(-2, 3, (rows, Hq + 2 * Hkv, hd // 32, 32)) * 2.0 ** -149
    top = rng.integers(0, 10, x.shape[:3])
    x[top == 0] = 0
    x[..., 3] = top * 2.0 ** -149 * rng.choice([-1, 1], top.shape)
    x[0, ..., 3] = [[1 * 2.0 ** -149]] * x.shape[1]
    x[1, ..., 3] = [[3 * 2.0 ** -149]] * x.shape[1]
    x[0, ..., 4:], x[1, ..., 4:], x[:2, ..., :3] = 0, 0, 0
    x = x.astype(np.float32).reshape(rows, -1)
    cos, sin = np.ones((4, hd // 2), np.float32), np.zeros((4, hd // 2), np.float32)
    before, entry = noise(rng, 3, Hkv, hd), rng.permutation(3 * 64)[:rows]
    _, cache = run_append("f32", x, x.shape[1], cos, sin, [1] * rows, entry, Hq, hd, before)
    want, h = before.copy(), x.astype(np.float64).reshape(rows, -1, hd)
    for r, e in enumerate(entry):
        put(want[e // 64], e % 64, quantise(h[r, Hq:Hq + Hkv]), quantise(h[r, Hq + Hkv:]))
    assert quantise(h[0])[1].min() == quantise(h[1])[1].min() == 2.0 ** -23
    assert np.array_equal(canonical(cache), canonical(want))


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
@pytest.mark.parametrize("Hkv,hd,rows", [(8, 128, 1), (2, 64, 5), (3, 128, 64), (1, 64, 200), (5, 128, 333),
                                         (40, 64, 130)])
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


# ------------------------------------------------------------------ attention: what may be in the data

# heads and rows of a prompt that take 16-row items, and that take tiles (16-bit types)
FEW, MANY = (8, 2), (32, 16)


@gpu
@pytest.mark.parametrize("dtype,hd", [("f16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("heads", [FEW, MANY])
def test_missing_blocks_slots_and_positions(dtype, hd, heads):
    """Missing blocks (-1 and past the pool) are left out of a row's keys; slots
    outside the table and negative positions give zeros; contexts are clamped to max_ctx."""
    rng = np.random.default_rng(5)
    Hq, Hkv = heads
    b = Batch(rng, dtype, Hkv, hd, [500, 300, 260, 210, 150])
    b.table[b.slot[0], [1, 5]] = -1, b.n_blocks
    b.table[b.slot[1], 3:] = -7
    b.table[b.slot[3], :] = -1
    rows = [(0, 499), (1, 299), (2, 259), (3, -1), (3, 209), (4, 149), (2, 255)]
    q = values(rng, (len(rows), Hq, hd), dtype)
    slots = [b.slot[j] for j, _ in rows]
    slots[6] = b.table.shape[0]
    got = run_decode(b, q, rows, Hq, max_ctx=490, slots=slots)
    gone = {0: [(64, 128), (320, 384)], 1: [(192, 300)], 2: [], 3: [(0, 210)], 4: []}
    seqs = [(0, 370, 130), (1, 200, 95), (4, 140, 10)]
    q2 = values(rng, (sum(x for _, _, x in seqs), Hq, hd), dtype)
    got2 = run_prefill(b, q2, seqs, Hq, max_ctx=490, slots=[b.slot[0], b.slot[1], -1])

    def check(qr, have, j, p):
        keep = np.array([i for i in range(min(p + 1, 490)) if not any(lo <= i < hi for lo, hi in gone[j])], dtype=int)
        if not len(keep):
            assert np.all(have == 0), (j, p)
            return
        K, V = b.K[j][keep], b.V[j][keep]
        args = ([p], np.arange(len(keep)), Hkv)
        ref, mag = (T.attention(qr, K, v, *args) for v in (V, np.abs(V)))
        assert np.all(np.abs(have - ref) <= bound(dtype, qr, K, V, ref, mag)), (j, p)

    for m, (j, p) in enumerate(rows):
        if m in (3, 6):
            assert np.all(got[m] == 0)
        else:
            check(q[m:m + 1], got[m:m + 1], j, p)
    assert np.all(got2[225:] == 0)
    for r in range(0, 225, 3):
        j, p = (0, 370 + r) if r < 130 else (1, 200 + r - 130)
        check(q2[r:r + 1], got2[r:r + 1], j, p)


@gpu
@pytest.mark.parametrize("dtype,hd", [("f16", 128), ("bf16", 64), ("f32", 64), ("bf16", 128)])
@pytest.mark.parametrize("heads", [FEW, MANY])
def test_nan_groups_reach_the_rows_that_see_them(dtype, hd, heads):
    """A group that held an infinity reads as NaN: rows before its position keep
    their results to the bit, those from there on get NaN, of K in all dims of
    its head, of V in the group's dims alone."""
    rng = np.random.default_rng(6)
    Hq, Hkv = heads
    G, n, bad = Hq // Hkv, 190, 107
    b = Batch(rng, dtype, Hkv, hd, [n, 140])
    q = values(rng, (n + 40, Hq, hd), dtype)
    seqs = [(0, 0, n), (1, 100, 40)]
    clean = run_prefill(b, q, seqs, Hq)
    check_prefill(b, q, clean, seqs)
    kb, vb, half, ks, vs = byte_tables(hd)
    blk, p = b.bytes[b.table[b.slot[0], bad // 64]], bad % 64
    blk[0, [ks[p, 1], ks[p, 1] + 1]] = 0x00, 0x7E
    blk[1, [vs[p, 1], vs[p, 1] + 1]] = 0x00, 0x7E
    got = run_prefill(b, q, seqs, Hq)
    dec = run_decode(b, q[:3], [(0, bad - 1), (0, bad), (0, n - 1)], Hq)
    assert np.array_equal(got[:bad], clean[:bad]) and np.array_equal(got[n:], clean[n:])
    ref, tol = b.reference(q[:1], 0, [bad - 1])
    assert np.all(np.abs(dec[:1] - ref) <= tol)
    keep = np.arange(hd) // 32 != 1
    for rows, was in ((got[bad:n], clean[bad:n]), (dec[1:], None)):
        assert np.isnan(rows[:, :G]).all() and np.isnan(rows[:, G:2 * G][..., ~keep]).all()
        assert np.isfinite(rows[:, 2 * G:]).all() and np.isfinite(rows[:, G:2 * G][..., keep]).all()
        if was is not None:
            assert np.array_equal(rows[:, 2 * G:], was[:, 2 * G:])
            assert np.array_equal(rows[:, G:2 * G][..., keep], was[:, G:2 * G][..., keep])


@gpu
@pytest.mark.parametrize("dtype,heads,seq", [
    ("f16", (32, 8), (1500, 1)), ("bf16", (32, 8), (1500, 30)), ("f32", (4, 4), (1500, 9)),
    ("bf16", (64, 8), (2016, 100)), ("f16", (64, 8), (2016, 100)), ("f16", (32, 8), (90, 3)),
    ("bf16", (64, 8), (0, 120))])
def test_nan_scores_make_nan_rows(dtype, heads, seq):
    """A row of q that holds NaN, and a key that does and is alone in its block, the last."""
    rng = np.random.default_rng(77)
    Hq, Hkv = heads
    hd, cached, new = 128, *seq
    n = cached + new
    n += (1 - n) % 64               # the last key begins a block
    cached = n - new
    b = Batch(rng, dtype, Hkv, hd, [n])
    q = values(rng, (new, Hq, hd), dtype)
    if new > 1:
        q[0] = np.nan
        got = run_prefill(b, q, [(0, cached, new)], Hq)
        assert np.isnan(got[0]).all() and np.isfinite(got[1:]).all()
    dec = run_decode(b, np.full((1, Hq, hd), np.nan), [(0, n - 1)], Hq)
    assert np.isnan(dec).all()
    q[0] = 1.0
    k = rng.standard_normal((Hkv, hd))
    k[:, 40] = np.nan
    b.store(b.slot[0], n - 1, quantise(k), quantise(rng.standard_normal((Hkv, hd))))
    dec = run_decode(b, q[:1], [(0, n - 1)], Hq)
    assert np.isnan(dec).all()
    if new > 1:
        got = run_prefill(b, q, [(0, cached, new)], Hq)
        assert np.isnan(got[-1]).all() and np.isfinite(got[:-1]).all()


@gpu
@pytest.mark.parametrize("dtype,lo,hi", [("f16", 4, 30), ("bf16", 4, 90), ("f32", 4, 90)])
@pytest.mark.parametrize("many", [False, True])
def test_scores_of_any_size(dtype, lo, hi, many):
    """Scores from 2^lo to 2^hi, one size a head, each exact in fp32: the weights
    are right whatever the size, in decode, in 16-row items and in tiles."""
    rng = np.random.default_rng(hi)
    Hq = Hkv = 16 if many else 8
    hd, ctx = 64, [131, 200, 420, 130]
    b = Batch(rng, dtype, Hkv, hd, ctx)
    e = np.linspace(lo, hi, Hkv).astype(int)
    a = np.clip(e - 14, -8, 14 if dtype == "f16" else 80)     # q = 2^a, k = 6 m 2^(e - a - 14): 64 dims add 6 bits
    for j, c in enumerate(ctx):
        m = rng.integers(32, 64, (c, Hkv)) * rng.choice([-1.0, 1.0], (c, Hkv))
        k = np.repeat((6 * m * np.exp2(e - a - 14))[:, :, None], hd, axis=2)
        code = quantise(k)
        assert np.array_equal(held(*code), k)
        b.K[j] = k
        for p in range(c):
            v = quantise(b.V[j][p])
            b.store(b.slot[j], p, [x[p] for x in code], v)
            b.V[j][p] = held(*v)
    ones = lambda n: np.broadcast_to(np.exp2(a)[None, :, None], (n, Hq, hd)).copy()
    got = run_decode(b, ones(4), [(j, c - 1) for j, c in enumerate(ctx)], Hq)
    seqs = [(j, c - 100, 100) for j, c in enumerate(ctx)]
    pre = run_prefill(b, ones(400), seqs, Hq)
    u = UNIT[dtype]

    def check(have, j, p):
        args = ([p], np.arange(p + 1), Hkv)
        ref, mag = (T.attention(ones(1), b.K[j][:p + 1], v[:p + 1], *args) for v in (b.V[j], np.abs(b.V[j])))
        # the scores are exact: only weights (times scales), sums and the result are rounded; the scale 1/8 is
        # exact, its base-2 factor is not: 2^-23 of a score's distance from the largest, which weights that are not
        # yet 0 keep below 2^7
        tol = ((p + 97) * 2.0 ** -24 + 2.0 ** -15) * mag + 2.0 ** -24
        if dtype != "f32":
            tol = tol + (2.0 ** -11 * mag + u * np.abs(ref)) * 1.02 + (p + 1) * 2.0 ** -24 * np.abs(b.V[j]).max()
        else:
            tol = tol + 2.0 ** -24 * np.abs(ref)
        assert np.all(np.abs(have - ref) <= tol), (j, p, (np.abs(have - ref) / tol).max())

    for j, c in enumerate(ctx):
        check(got[j:j + 1], j, c - 1)
        for i in (0, 1, 50, 99):
            check(pre[100 * j + i:100 * j + i + 1], j, c - 100 + i)


@gpu
@pytest.mark.parametrize("dtype,hd", [("f16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("heads", [FEW, MANY])
@pytest.mark.parametrize("vscale", [2.0 ** -21, 1e-4, 9000.0])
def test_values_of_any_size(dtype, hd, heads, vscale):
    """V near the least numbers held and near the largest, and of sizes that differ from place to place."""
    rng = np.random.default_rng(hd)
    Hq, Hkv = heads
    ctx = [200, 77]
    spread = np.exp2(rng.integers(-4, 1, (200, 1, 1)))
    b = Batch(rng, dtype, Hkv, hd, ctx)
    for j, c in enumerate(ctx):
        v = quantise(rng.standard_normal((c, Hkv, hd)) * vscale * spread[:c])
        b.V[j] = held(*v)
        k = quantise(b.K[j])
        b.K[j] = held(*k)
        for p in range(c):
            b.store(b.slot[j], p, [x[p] for x in k], [x[p] for x in v])
    q = values(rng, (250, Hq, hd), dtype)
    seqs = [(0, 0, 200), (1, 27, 50)]
    got = run_prefill(b, q, seqs, Hq)
    dec = run_decode(b, q[:2], [(0, 199), (1, 76)], Hq)
    for have, pairs in ((got, [(r, 0, r) for r in range(200)] + [(200 + r, 1, 27 + r) for r in range(50)]),
                        (dec, [(0, 0, 199), (1, 1, 76)])):
        for r, j, p in pairs[::7] + pairs[-1:]:
            ref, tol = b.reference(q[r:r + 1], j, [p])
            if dtype == "f16":      # results below 2^-14 are rounded to steps of 2^-24
                tol = tol + 2.0 ** -25
            else:
                tol = tol - 2.0 ** -25 * (dtype == "bf16")
            assert np.all(np.abs(have[r:r + 1] - ref) <= tol), (j, p)


@gpu
@pytest.mark.parametrize("dtype,hd", [("f16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("heads", [FEW, MANY])
def test_large_values_beside_small_ones(dtype, hd, heads):
    """V's groups of sizes up to 2^12 apart, one of them 2^12 times larger still in one place.
    Bounds are of each group's own largest value, and 2^-39 of the largest of all a key (half
    the least step of fp16 where the largest scale is held as 2^14)."""
    rng = np.random.default_rng(hd + 5)
    Hq, Hkv = heads
    ctx = [200, 77]
    b = Batch(rng, dtype, Hkv, hd, ctx)
    size = np.exp2(-rng.integers(0, 13, (1, Hkv, hd // 32)).astype(float))
    size[:, :, 1] = 1.0
    for j, c in enumerate(ctx):
        large = np.ones((c, 1, hd // 32))
        large[20, :, 1] = 2.0 ** 12
        v = quantise(rng.standard_normal((c, Hkv, hd)) * np.repeat(size * large, 32, axis=2))
        b.V[j] = held(*v)
        k = quantise(b.K[j])
        b.K[j] = held(*k)
        for p in range(c):
            b.store(b.slot[j], p, [x[p] for x in k], [x[p] for x in v])
    q = values(rng, (250, Hq, hd), dtype)
    got = run_prefill(b, q, [(0, 0, 200), (1, 27, 50)], Hq)
    dec = run_decode(b, q[:2], [(0, 199), (1, 76)], Hq)
    for have, pairs in ((got, [(r, 0, r) for r in range(200)] + [(200 + r, 1, 27 + r) for r in range(50)]),
                        (dec, [(0, 0, 199), (1, 1, 76)])):
        for r, j, p in pairs[::7] + pairs[-1:]:
            K, V, qr = b.K[j][:p + 1], b.V[j][:p + 1], q[r:r + 1]
            ref, mag = (T.attention(qr, K, v, [p], np.arange(p + 1), Hkv) for v in (V, np.abs(V)))
            for h in range(Hkv):
                for d in range(0, hd, 32):
                    at = (slice(None), slice(h * Hq // Hkv, (h + 1) * Hq // Hkv), slice(d, d + 32))
                    tol = bound(dtype, qr, K, V[:, h:h + 1, d:d + 32], ref[at], mag[at])
                    tol = tol + (p + 1) * 2.0 ** -39 * np.abs(V).max() - 2.0 ** -25 * (dtype == "bf16")
                    assert np.all(np.abs(have[r:r + 1][at] - ref[at]) <= tol), (j, p, h, d)


@gpu
def test_bf16_queries_of_any_size():
    """Rows of q of very different sizes, and dims of very different sizes in a row, in tiles."""
    rng = np.random.default_rng(12)
    Hq, Hkv, hd = 32, 16, 128
    b = Batch(rng, "bf16", Hkv, hd, [150])
    q = values(rng, (150, Hq, hd), "bf16")
    size = np.exp2(rng.integers(-100, 1, (150, Hq, 1)).astype(float))
    wide = np.exp2(-rng.integers(0, 60, (150, Hq, hd)).astype(float))
    wide[:, ::2] = 1.0
    q = torch.from_numpy(q * size * wide).bfloat16().double().numpy()
    q[7] = 0
    got = run_prefill(b, q, [(0, 0, 150)], Hq)
    for r in range(0, 150, 7):      # each row's bound is of its own size
        for h in range(0, Hq, 5):
            K, V = b.K[0][:r + 1, h // 2:h // 2 + 1], b.V[0][:r + 1, h // 2:h // 2 + 1]
            qr = q[r:r + 1, h:h + 1]
            ref, mag = (T.attention(qr, K, v, [r], np.arange(r + 1), 1) for v in (V, np.abs(V)))
            assert np.all(np.abs(got[r:r + 1, h:h + 1] - ref) <= bound("bf16", qr, K, V, ref, mag)), (r, h)


@gpu
@pytest.mark.parametrize("heads", [FEW, MANY])
def test_bf16_queries_near_the_largest_number(heads):
    """q at 2^127 along one dim, where K is equal at all places but one: even weights, or that place alone."""
    rng = np.random.default_rng(13)
    Hq, Hkv = heads
    hd, n = 128, 150
    b = Batch(rng, "bf16", Hkv, hd, [n])
    K = np.full((n, Hkv, hd), 6 * 2.0 ** -11)
    K[:, :, 0] = 2.0 ** -11
    K[40, :, 0] = 1.5 * 2.0 ** -11
    k, v = quantise(K), quantise(b.V[0])
    assert np.array_equal(held(*k), K)
    for p in range(n):
        b.store(b.slot[0], p, [x[p] for x in k], [x[p] for x in v])
    q = np.zeros((n, Hq, hd))
    q[:, :, 0] = 2.0 ** 127
    got = run_prefill(b, q, [(0, 0, n)], Hq)
    V = np.repeat(held(*v), Hq // Hkv, axis=1)
    for r in (0, 20, 39, 40, 41, 149):
        ref = V[:r + 1].mean(0) if r < 40 else V[40]
        # weights and the result rounded to 11 and 8 bits, sums of 41 terms in 24
        mag = np.abs(V[:r + 1]).mean(0) if r < 40 else np.abs(ref)
        assert np.all(np.abs(got[r] - ref) <= (2.0 ** -11 + 2.0 ** -19) * mag + 2.0 ** -8 * np.abs(ref) * 1.01), r


def one_dim_batch(rng, dtype, Hkv, n, base, at_40):
    """A sequence whose K differs along dim 0 alone: `base` codes' worth there, at place 40 `at_40`."""
    b = Batch(rng, dtype, Hkv, 128, [n])
    K = np.full((n, Hkv, 128), 6 * 2.0 ** -11)
    K[:, :, 0] = base * 2.0 ** -11
    K[40, :, 0] = at_40 * 2.0 ** -11
    k, v = quantise(K), quantise(b.V[0])
    assert np.array_equal(held(*k), K)
    for p in range(n):
        b.store(b.slot[0], p, [x[p] for x in k], [x[p] for x in v])
    b.K[0], b.V[0] = K, held(*v)
    return b


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [FEW, MANY])
@pytest.mark.parametrize("n", [150, 1500])
@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** 125, 2.0 ** 127 * 1.5, (2 - 2.0 ** -12) * 2.0 ** 127, -2.0 ** 127])
def test_queries_whose_products_with_codes_pass_fp32(dtype, heads, n, size):
    """q near the largest number along one dim, where K has codes up to 6: even weights as
    long as all places have the same, then that place alone which has the most."""
    rng = np.random.default_rng(14)
    Hq, Hkv = heads
    size = float(np.clip(size, None, (2 - 2.0 ** -7) * 2.0 ** 127)) if dtype == "bf16" else size
    least = size < 0                # then the least is the largest score
    b = one_dim_batch(rng, dtype, Hkv, n, 6 if least else 4, 4 if least else 6)
    q = np.zeros((n, Hq, 128))
    q[:, :, 0] = size
    q[:, :, 1] = 1.0                # of no account beside it
    got = run_prefill(b, q[:100], [(0, 0, 100)], Hq)
    dec = run_decode(b, q[:3], [(0, 39), (0, 40), (0, n - 1)], Hq)
    V = np.repeat(b.V[0], Hq // Hkv, axis=1)
    for have, p in [(got[r], r) for r in (0, 20, 39, 40, 41, 99)] + list(zip(dec, (39, 40, n - 1))):
        ref = V[:p + 1].mean(0) if p < 40 else V[40]
        mag = np.abs(V[:p + 1]).mean(0) if p < 40 else np.abs(ref)
        # weights and the result rounded to 11 and 8 bits, or neither; sums of 40 terms in 24
        half = 2.0 ** -24 * np.abs(ref) if dtype == "f32" else 2.0 ** -11 * mag + 2.0 ** -8 * np.abs(ref) * 1.01
        tol = 2.0 ** -18 * mag + half
        assert np.all(np.abs(have - ref) <= tol), p


@gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("heads", [FEW, MANY])
@pytest.mark.parametrize("n", [150, 1500])
def test_rows_of_scores_of_minus_infinity_are_zeros(dtype, heads, n):
    """An infinity in a row of q, of the sign that K does not have there: every score is
    minus infinity and the result 0; of K's sign it is NaN; the rows beside are as ever."""
    rng = np.random.default_rng(15)
    Hq, Hkv = heads
    b = one_dim_batch(rng, dtype, Hkv, n, 4, 6)
    q = values(rng, (100, Hq, 128), dtype)
    clean = run_prefill(b, q, [(0, n - 100, 100)], Hq)
    q[[3, 50], :, 0] = -np.inf
    q[70, :, 0] = np.inf
    got = run_prefill(b, q, [(0, n - 100, 100)], Hq)
    dec = run_decode(b, q[[3, 70]], [(0, n - 1)] * 2, Hq)
    assert np.all(got[[3, 50]] == 0) and np.all(dec[0] == 0)
    assert np.isnan(got[70]).all() and np.isnan(dec[1]).all()
    rest = np.setdiff1d(np.arange(100), [3, 50, 70])
    assert np.array_equal(got[rest], clean[rest])


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd", [("f16", 32, 8, 128), ("bf16", 8, 8, 64), ("f32", 16, 8, 128),
                                             ("f32", 8, 8, 64)])
@pytest.mark.parametrize("rows,ctx", [(1, 200), (3, 700), (5, 600), (8, 600), (12, 700), (1, 1500), (2, 1500),
                                      (4, 1500)])
def test_decode_of_few_blocks_and_many(dtype, Hq, Hkv, hd, rows, ctx):
    """Batches from 32 blocks and heads to over 1,000, of one item a row and of several."""
    rng = np.random.default_rng(rows + ctx)
    b = Batch(rng, dtype, Hkv, hd, [ctx - 13 * j for j in range(rows)])
    q = values(rng, (rows, Hq, hd), dtype)
    pairs = [(j, ctx - 13 * j - 1) for j in range(rows)]
    got = run_decode(b, q, pairs, Hq)
    for r, (j, p) in enumerate(pairs):
        ref, tol = b.reference(q[r:r + 1], j, [p])
        assert np.all(np.abs(got[r:r + 1] - ref) <= tol), (j, p)


# ------------------------------------------------------------------ attention: shapes of batches

@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,n", [("f16", 8, 2, 128, 40), ("bf16", 16, 16, 64, 45), ("f32", 24, 1, 64, 12),
                                               ("f16", 40, 1, 128, 33), ("bf16", 10, 5, 128, 300)])
def test_decode_batches_of_odd_rows(dtype, Hq, Hkv, hd, n):
    """Rows that share slots, in any order, of any position, with padding between; max_ctx above all contexts."""
    rng = np.random.default_rng(n)
    b = Batch(rng, dtype, Hkv, hd, [300, 64, 1, 129])
    rows = [(m % 4, [-1, 0, 63, 64, 127, 128, 299][m * 3 % 7]) for m in range(n)]
    rows = [(j, min(p, b.ctx[j] - 1)) for j, p in rows]
    q = values(rng, (n, Hq, hd), dtype)
    for top in (300, 320):
        b.table = np.pad(b.table, ((0, 0), (0, max(0, 5 - b.table.shape[1]))), constant_values=-1)
        got = run_decode(b, q, rows, Hq, max_ctx=top)
        for m, (j, p) in enumerate(rows):
            if p < 0:
                assert np.all(got[m] == 0)
            else:
                ref, tol = b.reference(q[m:m + 1], j, [p])
                assert np.all(np.abs(got[m:m + 1] - ref) <= tol), m


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [FEW, MANY])
def test_prefill_of_a_padded_batch(dtype, heads):
    """150 places for sequences of which five have rows, the others none and no slot."""
    rng = np.random.default_rng(150)
    (Hq, Hkv), hd = heads, 64
    new = np.zeros(150, int)
    new[[3, 63, 64, 100, 149]] = [40, 1, 33, 70, 9]
    b = Batch(rng, dtype, Hkv, hd, [90 + n if n else 0 for n in new])
    q = values(rng, (new.sum() + 4, Hq, hd), dtype)
    seqs = [(j, 90, n) for j, n in enumerate(new)]
    got = run_prefill(b, q, seqs, Hq, tail=4, slots=[s if n else -1 for s, n in zip(b.slot, new)])
    assert np.all(got[-4:] == 7)
    check_prefill(b, q, got, seqs)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_prefill_of_few_rows_among_many_empty_places(dtype):
    """16 rows of five sequences among 2^20 places, as a step of fixed size may hold."""
    rng = np.random.default_rng(20)
    Hq, Hkv, hd, places = 32, 8, 128, 1 << 20
    at, new, ctx = [0, 5, 64, 70000, places - 1], [1, 6, 1, 3, 5], [130, 76, 71, 73, 200]
    b = Batch(rng, dtype, Hkv, hd, ctx)
    q = values(rng, (16, Hq, hd), dtype)
    n, slot, pos = np.zeros(places, int), np.full(places, -1), np.full(places, -1)
    n[at], slot[at], pos[at] = new, b.slot, np.subtract(ctx, new)
    start, qd = i32(np.concatenate([[0], np.cumsum(n)])), torch.from_numpy(q).to(TYPES[dtype]).to(DEV)
    for max_new in (1, 6):                # one row a sequence, and all
        out = torch.full_like(qd, 7.0)
        ws = torch.empty(lp.kv4_prefill_attention_ws_bytes(16, Hq, Hkv, hd, 200), dtype=torch.uint8, device=DEV)
        lp.op_kv4_prefill_attention(qd, out, b.cache(), i32(b.table), start, i32(slot), i32(pos), max_new, 200, ws)
        got, r = out.double().cpu().numpy(), 0
        for j, (x, c) in enumerate(zip(new, ctx)):
            rows = min(x, max_new)
            ref, tol = b.reference(q[r:r + rows], j, np.arange(c - x, c - x + rows))
            assert np.all(np.abs(got[r:r + rows] - ref) <= tol), j
            r += x


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("heads", [FEW, MANY])
def test_rows_past_max_new_and_outside_the_rows(dtype, heads):
    """Of a sequence with more rows than max_new the first max_new are right, and
    those of the next sequences; entries of seq_start below 0 and above the rows
    count as these; a negative seq_pos is no row with keys."""
    rng = np.random.default_rng(8)
    (Hq, Hkv), hd = heads, 64
    b = Batch(rng, dtype, Hkv, hd, [190, 120, 160])
    q = values(rng, (112, Hq, hd), dtype)
    got = run_prefill(b, q, [(0, 100, 90), (1, 100, 20)], Hq, max_new=40, tail=2)
    for j, r, n in ((0, 0, 40), (1, 90, 20)):
        ref, tol = b.reference(q[r:r + n], j, np.arange(100, 100 + n))
        assert np.all(np.abs(got[r:r + n] - ref) <= tol)
    assert np.all(got[110:] == 7)
    n = 50
    for max_new in (n, 100):
        out = torch.full((n, Hq, hd), 7.0, dtype=TYPES[dtype], device=DEV)
        ws = torch.empty(max(16, lp.kv4_prefill_attention_ws_bytes(n, Hq, Hkv, hd, 160)), dtype=torch.uint8, device=DEV)
        lp.op_kv4_prefill_attention(torch.from_numpy(q[:n]).to(TYPES[dtype]).to(DEV), out, b.cache(), i32(b.table),
                                    i32([-9, 12, 30, 70, 90]), i32([b.slot[0], b.slot[1], b.slot[2], b.slot[0]]),
                                    i32([100, -3, 120, 5]), max_new, 160, ws)
        have = out.double().cpu().numpy()
        for j, r0, r1, p in ((0, 0, 12, 100), (2, 30, 50, 120)):
            ref, tol = b.reference(q[r0:r1], j, np.arange(p, p + r1 - r0))
            assert np.all(np.abs(have[r0:r1] - ref) <= tol), j
        assert np.all(have[12:30] == 0)


@gpu
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads", [FEW, (4, 4), MANY])
@pytest.mark.parametrize("after", [2, 22])
def test_places_past_max_new_cost_no_bits(hd, heads, after):
    """Positions that only rows from max_new on would see hold the largest values, the
    others some 2^-18: results are as near as ever, so near as weights of 11 bits make them."""
    rng = np.random.default_rng(18)
    (Hq, Hkv), first, new = heads, 150, 18
    b = Batch(rng, "bf16", Hkv, hd, [first + new], vscale=2.0 ** -18)
    for p in range(first + new, first + new + after):
        b.store(b.slot[0], p, *(quantise(rng.standard_normal((Hkv, hd)) * x) for x in (1.0, 3e4)))
    q = values(rng, (new + after, Hq, hd), "bf16")
    got = run_prefill(b, q, [(0, first, new + after)], Hq, max_new=new)
    ref, tol = b.reference(q[:new], 0, np.arange(first, first + new))
    tol = tol - 2.0 ** -25      # bf16 has no least step there
    assert np.all(np.abs(got[:new] - ref) <= tol), (np.abs(got[:new] - ref) / tol).max()


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_many_rows_that_no_sequence_has(dtype):
    """A batch of 3,000 rows of which sequences have three: its plan stays inside its workspace."""
    rng = np.random.default_rng(2)
    Hq, Hkv, hd = 32, 8, 64
    b = Batch(rng, dtype, Hkv, hd, [2000, 700])
    q = values(rng, (3000, Hq, hd), dtype)
    got = run_prefill(b, q, [(0, 1998, 2), (1, 699, 1)], Hq, start=1, tail=2996)
    check_prefill(b, q, got, [(0, 1998, 2), (1, 699, 1)], 1)
    assert np.all(got[0] == 7) and np.all(got[4:] == 7)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_walks_of_more_than_64_blocks(dtype):
    """All blocks of a row in one item, 71 of them: decode, and prompts in 16-row items (fp32) and tiles (fp16)."""
    rng = np.random.default_rng(64)
    hd, c = 64, 4540
    b = Batch(rng, dtype, 8, hd, [c])
    rows = [(0, c - 1 - 13 * m) for m in range(260)]
    q = values(rng, (260, 8, hd), dtype)
    got = run_decode(b, q, rows, 8)
    for m in (0, 1, 130, 259):
        ref, tol = b.reference(q[m:m + 1], 0, [rows[m][1]])
        assert np.all(np.abs(got[m:m + 1] - ref) <= tol), m
    seqs = [(0, c - 3 - 11 * m, 3) for m in range(270)]
    q = values(rng, (810, 8, hd), dtype)
    got = run_prefill(b, q, seqs, 8)
    for m in (0, 7, 269):
        ref, tol = b.reference(q[3 * m:3 * m + 3], 0, list(range(seqs[m][1], seqs[m][1] + 3)))
        assert np.all(np.abs(got[3 * m:3 * m + 3] - ref) <= tol), m


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_one_row_of_more_than_64_parts(dtype):
    rng = np.random.default_rng(65)
    c = 64 * 4 * 66 + 5
    b = Batch(rng, dtype, 1, 64, [c])
    q = values(rng, (2, 2, 64), dtype)
    got = run_decode(b, q, [(0, c - 1), (0, 3000)], 2)
    for m, p in enumerate((c - 1, 3000)):
        ref, tol = b.reference(q[m:m + 1], 0, [p])
        assert np.all(np.abs(got[m:m + 1] - ref) <= tol)
    got = run_prefill(b, q, [(0, c - 2, 2)], 2)
    check_prefill(b, q, got, [(0, c - 2, 2)])


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_the_largest_batches_that_always_fit(dtype):
    """Rows times heads just under 2^22, of which some rows are looked at."""
    rng = np.random.default_rng(22)
    M, Hq, Hkv, hd, ctx = 65530, 64, 8, 64, [101, 228, 300]
    assert M * Hq < 1 << 22 <= (M + 8) * Hq
    b = Batch(rng, dtype, Hkv, hd, ctx)
    q = torch.randn(M, Hq, hd, generator=torch.Generator(DEV).manual_seed(1), device=DEV).to(TYPES[dtype])
    out, cache, table = torch.empty_like(q), b.cache(), i32(b.table)
    j = np.arange(M) % 3
    slot, pos = i32(b.slot[j]), i32(np.array(ctx)[j] - 1)
    some = [0, 1, 2, 4095, 32768, 60001, M - 2, M - 1]
    for f, size, index in ((lp.op_kv4_decode_attention, lp.kv4_decode_attention_ws_bytes, (slot, pos)),
                           (lp.op_kv4_prefill_attention, lp.kv4_prefill_attention_ws_bytes,
                            (i32(np.arange(M + 1)), slot, pos, 1))):
        out.fill_(7)
        ws = torch.empty(size(M, Hq, Hkv, hd, 300), dtype=torch.uint8, device=DEV)
        f(q, out, cache, table, *index, 300, ws)
        qs, have = q[some].double().cpu().numpy(), out[some].double().cpu().numpy()
        for i, m in enumerate(some):
            ref, tol = b.reference(qs[i:i + 1], j[m], [ctx[j[m]] - 1])
            assert np.all(np.abs(have[i:i + 1] - ref) <= tol), m


@gpu
def test_caches_past_4_gib():
    """Blocks whose byte offsets pass 32 bits: what a small cache gives, to the bit."""
    rng = np.random.default_rng(21)
    Hq, Hkv, hd = 16, 8, 128
    ctx = [201 + 40 * i for i in range(12)]
    b = Batch(rng, "f16", Hkv, hd, ctx)
    n = 59000                     # of 73,728 bytes
    big = torch.empty(n, Hkv, 72 * hd, dtype=torch.uint8, device=DEV)
    big[-b.n_blocks:] = b.cache()
    up = n - b.n_blocks
    small_cache, small_table = b.cache, b.table

    def call(f, *args):
        small = f(b, *args)
        b.cache, b.table, b.n_blocks = lambda: big, np.where(b.table >= 0, b.table + up, -1), n
        large = f(b, *args)
        b.cache, b.table, b.n_blocks = small_cache, small_table, n - up
        assert np.isfinite(small).all() and np.array_equal(small, large)

    q = values(rng, (700, Hq, hd), "f16")
    call(run_decode, q[:2], [(j, ctx[j] - 1) for j in range(2)], Hq)
    call(run_decode, q[:144], [(j, ctx[j] - 1) for j in range(12)] * 12, Hq)
    call(run_prefill, q[:100], [(0, 200, 1), (11, 300, 99)], Hq)
    call(run_prefill, q[:600], [(j, 100, 50) for j in range(12)], Hq)
    # append at the last places and read them back, into an ordinary cache past 4 GiB too
    rows, m = 65, 34000
    entry = torch.arange(n * 64 - 70, n * 64 - 5, dtype=torch.int64, device=DEV)
    x = rng.standard_normal((rows, (Hq + 2 * Hkv) * hd)).astype(np.float32)
    cos, sin = np.ones((4, hd // 2), np.float32), np.zeros((4, hd // 2), np.float32)
    qd = torch.empty(rows, Hq, hd, dtype=torch.float16, device=DEV)
    lp.op_kv4_append(torch.from_numpy(x).to(DEV), torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV),
                     i32([1] * rows), entry, qd, big)
    kc = torch.empty(m, Hkv, 64, hd, dtype=torch.float16, device=DEV)
    vc = torch.empty(m, Hkv, hd, 64, dtype=torch.float16, device=DEV)
    to = torch.arange(m * 64 - 66, m * 64 - 1, dtype=torch.int64, device=DEV)
    lp.op_kv4_read(big, entry, to, kc, vc)
    torch.cuda.synchronize()
    h = x.reshape(rows, -1, hd)
    for r in (0, 1, 63, 64):
        blk, p = divmod(int(to[r]), 64)
        assert np.array_equal(kc[blk, :, p].double().cpu().numpy(), held(*quantise(h[r, Hq:Hq + Hkv])))
        assert np.array_equal(vc[blk, :, :, p].double().cpu().numpy(), held(*quantise(h[r, Hq + Hkv:])))


@gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_read_of_many_contexts(dtype):
    """Contexts block by block, one after the other in the list, with rows of no
    entry, a place left out and a context that starts inside a block among them."""
    rng = np.random.default_rng(44)
    Hkv, hd, n_blocks = 40, 128, 60
    cache = noise(rng, n_blocks, Hkv, hd)
    for lo in (32 * hd, 68 * hd):
        s = scales(np.abs(rng.standard_normal((n_blocks, Hkv, 2 * hd))))
        cache[:, :, lo:lo + 4 * hd] = s.astype(np.float16).view(np.uint8)
    free, src, dst, at = rng.permutation(n_blocks), [], [], 0
    for c in (130, 64, 1, 300, 63, 192, 129):
        blocks, free = free[:ceil64(c)], free[ceil64(c):]
        p = np.arange(c)
        src += (blocks[p // 64] * 64 + p % 64).tolist() + [-1] * (c % 3)
        dst += (at + p).tolist() + [-1] * (c % 3)
        at += ceil64(c) * 64
    src, dst = np.array(src), np.array(dst)
    src[200], dst[333] = -1, 1 << 40
    p = np.arange(70)                     # from the middle of a block to the middle of one
    src, dst = np.append(src, free[0] * 64 + 5 + p % 50), np.append(dst, at + 9 + p)
    n_dst = at // 64 + 2
    kc = torch.full((n_dst, Hkv, 64, hd), 7.0, dtype=TYPES[dtype], device=DEV)
    vc = torch.full((n_dst, Hkv, hd, 64), 7.0, dtype=TYPES[dtype], device=DEV)
    lp.op_kv4_read(torch.from_numpy(cache).to(DEV), i64(src), i64(dst), kc, vc)
    torch.cuda.synchronize()
    wk, wv = np.full(kc.shape, 7.0), np.full(vc.shape, 7.0)
    for s, d in zip(src, dst):
        if 0 <= s and 0 <= d < n_dst * 64:
            wk[d // 64, :, d % 64], wv[d // 64, :, :, d % 64] = get(cache[s // 64], s % 64)
    assert np.array_equal(kc.double().cpu().numpy(), wk) and np.array_equal(vc.double().cpu().numpy(), wv)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("over", [1, 2, 3, 30, 62])
@pytest.mark.parametrize("more", [0, 90])
def test_read_of_a_last_block_that_starts_anywhere(dtype, over, more):
    """The last whole block of a list starts `over` places past a multiple of 64 of
    the list, and nothing after it begins a block."""
    rng = np.random.default_rng(over)
    Hkv, hd, n_blocks = 40, 64, 30
    cache = noise(rng, n_blocks, Hkv, hd)
    for lo in (32 * hd, 68 * hd):
        s = scales(np.abs(rng.standard_normal((n_blocks, Hkv, 2 * hd))))
        cache[:, :, lo:lo + 4 * hd] = s.astype(np.float16).view(np.uint8)
    dst = np.concatenate([np.arange(12 * 64), 12 * 64 + 1 + np.arange(over), 13 * 64 + np.arange(64),
                          16 * 64 + rng.permutation([x for x in range(8 * 64) if x % 64])[:more]])
    src = rng.permutation(n_blocks)[dst // 64] * 64 + dst % 64
    n_dst = 24
    kc = torch.full((n_dst, Hkv, 64, hd), 7.0, dtype=TYPES[dtype], device=DEV)
    vc = torch.full((n_dst, Hkv, hd, 64), 7.0, dtype=TYPES[dtype], device=DEV)
    lp.op_kv4_read(torch.from_numpy(cache).to(DEV), i64(src), i64(dst), kc, vc)
    torch.cuda.synchronize()
    wk, wv = np.full(kc.shape, 7.0), np.full(vc.shape, 7.0)
    for s, d in zip(src, dst):
        wk[d // 64, :, d % 64], wv[d // 64, :, :, d % 64] = get(cache[s // 64], s % 64)
    assert np.array_equal(kc.double().cpu().numpy(), wk) and np.array_equal(vc.double().cpu().numpy(), wv)


# ------------------------------------------------------------------ graphs and streams

@gpu
def test_steps_in_captured_graphs():
    """Append, decode and read-back captured once, a prefill beside them with the
    same workspace, replayed in turn with eager work between, against eager results."""
    rng = np.random.default_rng(30)
    Hq, Hkv, hd, n = 32, 8, 128, 20
    b = Batch(rng, "f16", Hkv, hd, [960 + i for i in range(n)])
    cache, table, slot, top, new = b.cache(), i32(b.table), i32(b.slot), 1024, 30
    qp = torch.from_numpy(values(rng, (n * new, Hq, hd), "f16")).half().to(DEV)
    x = torch.from_numpy(rng.standard_normal((n, (Hq + 2 * Hkv) * hd)).astype(np.float32)).to(DEV)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in rope_tables(1100, hd))
    start, first = i32(np.arange(n + 1) * new), i32([900] * n)
    pos = [959 + i for i in range(n)]
    entry = i64([b.table[s, p // 64] * 64 + p % 64 for s, p in zip(b.slot, pos)])
    pos, to = i32(pos), i64(np.arange(n))
    ws = torch.empty(max(lp.kv4_decode_attention_ws_bytes(n, Hq, Hkv, hd, top),
                         lp.kv4_prefill_attention_ws_bytes(n * new, Hq, Hkv, hd, top)), dtype=torch.uint8, device=DEV)
    qd = torch.zeros(n, Hq, hd, dtype=torch.float16, device=DEV)
    outs = [torch.zeros_like(qp), torch.zeros_like(qd)]
    kc = torch.zeros(1, Hkv, 64, hd, dtype=torch.float16, device=DEV)
    vc = torch.zeros(1, Hkv, hd, 64, dtype=torch.float16, device=DEV)

    def prefill():
        lp.op_kv4_prefill_attention(qp, outs[0], cache, table, start, slot, first, new, top, ws)

    def decode():
        lp.op_kv4_append(x, cos, sin, pos, entry, qd, cache)
        lp.op_kv4_decode_attention(qd, outs[1], cache, table, slot, pos, top, ws)
        lp.op_kv4_read(cache, entry, to, kc, vc)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (*outs, qd, kc, vc, cache)]

    decode()                # the appended rows stay the same from here on
    prefill()
    want, graphs = results(), []
    for f in (prefill, decode):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            f()
        graphs.append(graph)
    for _ in range(4):
        for t in (*outs, qd, kc, vc):
            t.fill_(9)
        want_k = want[3].clone()
        want_k[:, :, n:] = 9
        want_v = want[4].clone()
        want_v[..., n:] = 9
        for k in (0, 1):
            ws.random_(0, 256)
            graphs[k].replay()
        have = results()
        assert torch.equal(have[0], want[0]) and torch.equal(have[1], want[1]) and torch.equal(have[2], want[2])
        assert torch.equal(have[3], want_k) and torch.equal(have[4], want_v) and torch.equal(have[5], want[5])
        assert torch.isfinite(have[0]).all() and torch.isfinite(have[1]).all()
        torch.ones(1000, device=DEV).sum().item()


@gpu
def test_two_streams_at_once():
    """The same calls on two streams with workspaces of their own, many times over, give what one gives alone."""
    rng = np.random.default_rng(3)
    Hq, Hkv, hd, ctx = 32, 8, 128, [701 + 40 * i for i in range(16)]
    b = Batch(rng, "f16", Hkv, hd, ctx)
    q = [torch.from_numpy(values(rng, (16, Hq, hd), "f16")).half().to(DEV) for _ in range(2)]
    cache, slot, pos, table, top = b.cache(), i32(b.slot), i32([c - 1 for c in ctx]), i32(b.table), max(ctx)
    nb = lp.kv4_decode_attention_ws_bytes(16, Hq, Hkv, hd, top)

    def call(k, out, ws):
        lp.op_kv4_decode_attention(q[k], out, cache, table, slot, pos, top, ws)

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


# ------------------------------------------------------------------ refusals (no GPU is touched)

F16, F32, OK, EINVAL = lp.LP_F16, lp.LP_F32, lp.LP_OK, lp.LP_EINVAL
A = 1 << 20  # an aligned address that is never read: every call below returns before a launch


def test_cache_bytes():
    f = lp.lib().lp_op_kv4_cache_bytes
    assert f(7, 8, 128) == 7 * 8 * 9216 and f(1, 1, 64) == 4608 and f(1 << 33, 40, 128) == (1 << 33) * 40 * 9216
    assert f(0, 8, 128) == f(7, 0, 128) == f(7, 8, 96) == f(-1, 8, 64) == 0


def test_append_refusals():
    f = lp.lib().lp_op_kv4_append
    names = ("dtype", "qkv", "ld", "cos", "sin", "n_pos", "pos", "entry", "rows", "q", "cache", "n_blocks", "Hq", "Hkv",
             "hd", "stream")
    good = [F16, A, 1536, A, A, 100, A, A, 3, A, A, 5, 8, 2, 128, None]

    def call(**bad):
        return f(*[bad.get(k, v) for k, v in zip(names, good)])

    assert call(rows=0) == OK
    assert call(rows=0, qkv=None, cos=None, sin=None, pos=None, entry=None, q=None, cache=None) == OK
    for bad in (dict(dtype=7), dict(ld=1534), dict(ld=1537), dict(n_pos=0), dict(rows=-1), dict(n_blocks=0), dict(Hq=9),
                dict(Hkv=0), dict(hd=96)):
        assert call(**bad) == EINVAL, bad
        assert call(**{"rows": 0, **bad}) == EINVAL, bad
    for k in ("qkv", "cos", "sin", "pos", "entry", "q", "cache"):
        assert call(**{k: None}) == EINVAL, k
    for bad in (dict(qkv=A + 4), dict(cos=A + 4), dict(sin=A + 4), dict(q=A + 8), dict(cache=A + 8), dict(rows=700000)):
        assert call(**bad) == EINVAL, bad


def test_read_refusals():
    f = lp.lib().lp_op_kv4_read
    names = ("dtype", "cache", "n_blocks", "src", "dst", "rows", "k", "v", "n_dst", "Hkv", "hd", "stream")
    good = [F16, A, 5, A, A, 3, A, A, 6, 2, 128, None]

    def call(**bad):
        return f(*[bad.get(k, v) for k, v in zip(names, good)])

    pointers = ("cache", "src", "dst", "k", "v")
    assert call(rows=0) == OK and call(rows=0, **dict.fromkeys(pointers)) == OK
    for bad in (dict(dtype=7), dict(n_blocks=0), dict(rows=-1), dict(n_dst=0), dict(Hkv=0), dict(hd=80),
                dict(rows=1 << 26)):
        assert call(**bad) == EINVAL, bad
    for k in pointers:
        assert call(**{k: None}) == EINVAL, k
    for k in ("cache", "k", "v"):
        assert call(**{k: A + 8}) == EINVAL, k


@pytest.mark.parametrize("rows,Hkv", [(1, 1 << 24), (1, 1 << 26), (3, 1 << 24)])
def test_reads_past_one_launch_are_refused(rows, Hkv):
    """Rows times heads within their limit, but more workgroups than a launch has."""
    assert lp.lib().lp_op_kv4_read(F16, A, 5, A, A, rows, A, A, 6, Hkv, 128, None) == EINVAL
    assert "kv4 read: sizes" in lp.lib().lp_last_error(None).decode()


@pytest.mark.parametrize("decode", [True, False])
def test_attention_refusals(decode):
    L = lp.lib()
    f = L.lp_op_kv4_decode_attention if decode else L.lp_op_kv4_prefill_attention
    size = L.lp_op_kv4_decode_attention_ws_bytes if decode else L.lp_op_kv4_prefill_attention_ws_bytes
    head = dict(dtype=F16, q=A, out=A, cache=A, n_blocks=50, table=A, n_slots=4, wide=8)
    mid = dict(slot=A, pos=A, rows=4) if decode else dict(start=A, slot=A, pos=A, n=2, rows=40, max_new=30)
    tail = dict(Hq=8, Hkv=2, hd=128, max_ctx=500, ws=A, ws_bytes=1 << 40, stream=None)
    good = {**head, **mid, **tail}

    def call(**bad):
        return f(*[bad.get(k, v) for k, v in good.items()])

    pointers = [k for k in ("q", "out", "cache", "table", "start", "slot", "pos", "ws") if k in good]
    assert call(rows=0) == OK and call(**{"rows": 0, **dict.fromkeys(pointers)}) == OK
    if not decode:
        assert call(n=0) == OK and call(n=-1) == EINVAL and call(max_new=0) == EINVAL
    for bad in (dict(dtype=9), dict(rows=-1), dict(n_blocks=0), dict(n_slots=0), dict(wide=0), dict(wide=7), dict(Hq=9),
                dict(Hkv=0), dict(hd=80), dict(max_ctx=0), dict(max_ctx=(1 << 30) + 1), dict(rows=1 << 28)):
        assert call(**bad) == EINVAL, bad
        if "rows" not in bad:
            assert call(**{"rows": 0, **bad}) == EINVAL, bad
    for k in pointers:
        assert call(**{k: None}) == EINVAL, k
    for k in ("q", "out", "cache", "ws"):
        assert call(**{k: A + 8}) == EINVAL, k
    need = size(good["rows"], 8, 2, 128, 500)
    assert need > 0 and call(ws_bytes=need - 1) == EINVAL
    assert size(-1, 8, 2, 128, 500) == 0 and size(4, 8, 3, 128, 500) == 0 and size(4, 8, 2, 96, 500) == 0
    assert "kv4 attention" in L.lp_last_error(None).decode()


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("dtype", [F16, lp.LP_BF16, F32])
def test_work_past_one_launch_is_refused(decode, dtype):
    """Sizes within the limits each, whose workgroups together are too many."""
    L = lp.lib()
    f = L.lp_op_kv4_decode_attention if decode else L.lp_op_kv4_prefill_attention
    for rows, Hq, Hkv, ctx in ((1 << 21, 16, 16, 1), (1 << 25, 8, 8, 500), (1 << 29, 1, 1, 64)):
        seqs = [A, A, rows] if decode else [A, A, A, rows, rows, 1]
        assert f(dtype, A, A, A, 50, A, 4, 1 << 24, *seqs, Hq, Hkv, 64, ctx, A, 1 << 60, None) == EINVAL, rows
        assert "launch" in L.lp_last_error(None).decode()


@pytest.mark.parametrize("decode", [True, False])
def test_a_workspace_serves_smaller_steps(decode):
    """Sizes ascend with rows and contexts."""
    f = lp.kv4_decode_attention_ws_bytes if decode else lp.kv4_prefill_attention_ws_bytes
    rng = np.random.default_rng(1)
    for _ in range(2000):
        rows, ctx = int(np.exp(rng.uniform(0, 10))), int(np.exp(rng.uniform(0, 12)))
        Hkv, G = int(rng.integers(1, 41)), int(rng.integers(1, 20))
        less = f(int(rng.integers(1, rows + 1)), Hkv * G, Hkv, 128, int(rng.integers(1, ctx + 1)))
        assert 0 < less <= f(rows, Hkv * G, Hkv, 128, ctx)


def test_binding_refuses_tensors_that_do_not_fit():
    """Wrong devices, types, shapes and layouts raise before the library is called."""
    h = lambda *shape: torch.zeros(*shape, dtype=torch.float16)
    n = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    c = lambda *shape: torch.zeros(*shape, dtype=torch.uint8)
    e = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        lp.op_kv4_decode_attention(h(2, 4, 64), h(2, 4, 64), c(3, 2, 4608), n(2, 3), n(2), n(2), 70, c(64))
    with pytest.raises(ValueError, match="GPU"):
        lp.op_kv4_prefill_attention(h(2, 4, 64), h(2, 4, 64), c(3, 2, 4608), n(2, 3), n(2), n(1), n(1), 2, 70, c(64))
    with pytest.raises(ValueError, match="GPU"):
        lp.op_kv4_read(c(3, 2, 4608), e, e, h(3, 2, 64, 64), h(3, 2, 64, 64))
    with pytest.raises(ValueError, match="GPU"):
        lp.op_kv4_append(torch.zeros(2, 512), torch.zeros(9, 32), torch.zeros(9, 32), n(2), e, h(2, 4, 64),
                         c(3, 2, 4600))


@gpu
def test_binding_refuses_shapes_on_the_gpu():
    h = lambda *shape: torch.zeros(*shape, dtype=torch.float16, device=DEV)
    n = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=DEV)
    c = lambda *shape: torch.zeros(*shape, dtype=torch.uint8, device=DEV)
    e = torch.zeros(2, dtype=torch.int64, device=DEV)
    good = dict(q=h(2, 4, 64), out=h(2, 4, 64), cache=c(3, 2, 4608), block_table=n(2, 3), row_slot=n(2), row_pos=n(2),
                max_ctx=70, ws=c(1 << 20))
    lp.op_kv4_decode_attention(**good)
    for bad in (dict(q=h(2, 4, 128)[:, :, ::2]), dict(out=h(3, 4, 64)), dict(cache=c(3, 2, 4600)), dict(row_slot=n(3)),
                dict(row_pos=n(2).long()), dict(cache=h(3, 2, 4608)), dict(block_table=n(3, 2).T),
                dict(row_slot=n(2).cpu()),
                dict(cache=c(3, 2, 9216)), dict(q=h(2, 4, 80), out=h(2, 4, 80))):
        with pytest.raises(ValueError):
            lp.op_kv4_decode_attention(**{**good, **bad})
    with pytest.raises(lp.LPError):
        lp.op_kv4_decode_attention(**{**good, "max_ctx": 200})
    good = dict(cache=c(3, 2, 4608), src_entry=e, dst_entry=e, kc=h(2, 2, 64, 64), vc=h(2, 2, 64, 64))
    e.fill_(-1)
    lp.op_kv4_read(**good)
    for bad in (dict(dst_entry=e[:1]), dict(src_entry=e.int()), dict(vc=h(2, 2, 64, 32)), dict(kc=h(2, 3, 64, 64),
                vc=h(2, 3, 64, 64)), dict(vc=h(2, 2, 64, 64).float()), dict(cache=c(3, 2, 9216))):
        with pytest.raises(ValueError):
            lp.op_kv4_read(**{**good, **bad})
    torch.cuda.synchronize()


def test_loads_into_lds_keep_their_wait_states(tmp_path):
    """What is checked of the other kernels' loads into LDS, for these."""
    import test_device_code
    test_device_code.test_loads_into_lds_keep_their_wait_states("kv4_attention", tmp_path)
