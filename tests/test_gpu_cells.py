"""GPU parity of the operators around a 4-bit paged cache: the append (bytes equal to the definition's), its inverse (correctly rounded), norms and rotation, and
attention against plain 64-bit implementations at the sizes, layouts and masks where they can go wrong, and a run of them together.

Tolerances, element by element, with u half a step of the output's type (2^-11 fp16, 2^-8 bf16) and u16 = 2^-11.  Attention: weights w_j (summing to 1), cells
k_j = s_j c_j + z_j and v_j = s'_j c'_j + z'_j.  Of all kernels:
  * a weight exp2(x) has the error of its exponent: the score is made of 32-bit sums of 16-bit products of at most |q_i| (15 s + |z|), whose sum over i is Q
    ((D + 8) 2^-24 Q), scaled, biased and shifted in 32 bits (3 roundings of 2^-24 (|x| + |max|)), and exp2 itself 2^-22; it counts for the weight and for
    the sum that divides it:                                                              2 (ln 2 * that + 2^-22) A,  A = sum w_j |v_j|
  * 32-bit sums over n keys:                                                              2 n 2^-24 sum w_j (15 s'_j + |z'_j|)
  * the output's own rounding, u |out|, and half the smallest step where it is subnormal (fp16: 2^-25).
Up to 32 rows of a sequence and K/V head (codes are multiplied):
  * the matrix units keep a sum of eight products of codes, which are subnormal numbers in steps of 2^-20, to 2^-38 of the largest other factor: to
    2^-18 of a step.  In the score 2^-18 s sum |q_i|, in the result 2^-18 sum w_j s'_j
  * weights times scales are rounded to fp16, the codes' distance from 8 is what they multiply:   u16 sum w_j s'_j |c'_j - 8|, and 8 n 2^-39 max w_j s'_j for those
    below its normal range beside a largest of 2^8 or more.
More rows (values v are v 2^-e in fp16, with the largest of 32 s and 2^-14 |z| of a tile's keys, for V of all so far, between 2^e and 2^(e + 1); steps of at least 2^-24,
half of which is 2^-24 of the largest of 15 s and |z|, or less):
  * K and V are rounded: the score by u16 sum |q_i k_i| and 2^-24 max (15 s, |z|) sum |q_i|, the result by u16 A + 2^-24 max (15 s', |z'|)
  * weights are rounded, in the products and in the sum that divides them:                u16 (A + |out|), and n 2^-25 max |v|."""
import math
import random

import numpy as np
import pytest

import paper_2403_01136_amd as lpq
from test_gpu_paged import dtype_of, gen, ints, slopes_of

pytestmark = pytest.mark.gpu
U16 = 2.0**-11


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU (no fallback path)"
    lpq.load_library()


# ---- cells on the host, from the definition ----------------------------------------------------------------------------

def to_bits(x, dt):
    """float32 -> bits of the type, round to nearest even."""
    x = np.asarray(x, np.float32)
    if dt == "fp16":
        with np.errstate(over="ignore"):
            return x.astype(np.float16).view(np.uint16)
    b = x.view(np.uint32).astype(np.uint64)
    return np.where(np.isnan(x), 0x7fc0, (b + 0x7fff + (b >> 16 & 1)) >> 16).astype(np.uint16)


def of_bits(b, dt):
    b = np.asarray(b, np.uint16)
    return b.view(np.float16).astype(np.float32) if dt == "fp16" else (b.astype(np.uint32) << 16).view(np.float32)


def quantise(x, dt):
    """x float32 [d] -> (codes uint8 [d], scale bits, zero bits)."""
    nan = 0x7e00 if dt == "fp16" else 0x7fc0
    f = np.float32
    with np.errstate(over="ignore", invalid="ignore"):
        lo, hi = x.min(), x.max()
        scale = to_bits(f(f(hi - lo) / f(15)), dt)
        if not np.isfinite(x).all() or not np.isfinite(of_bits(scale, dt)):
            return np.zeros(len(x), np.uint8), nan, nan
        zero = f(lo + f(0))
        if scale == 0:
            return np.zeros(len(x), np.uint8), 0, int(to_bits(zero, dt))
        if np.isinf(of_bits(to_bits(f(15) * of_bits(scale, dt) + zero, dt), dt)):
            scale = scale - 1
        s = f(of_bits(scale, dt))
        codes = np.clip(np.rint((x - zero).astype(f) / s), 0, 15).astype(np.uint8)
    return codes, int(scale), int(to_bits(zero, dt))


def cell_bytes(codes, scale, zero):
    """(d / 2 bytes of codes, 4 bytes of parameters)."""
    words = np.zeros(len(codes) // 8, np.uint32)
    for e in range(8):
        words |= codes[e::8].astype(np.uint32) << np.uint32(4 * (e // 2) + 16 * (e % 2))
    return words.view(np.uint8), np.array([scale, zero], np.uint16).view(np.uint8)


def head_of(pages, page, h, d):
    """Views of one head of a page on the host: (codes [positions][d / 2], parameters [positions][4])."""
    g = pages[page, h].reshape(-1, 16 * (d // 2 + 4))
    return [(g[p // 16, p % 16 * (d // 2):(p % 16 + 1) * (d // 2)], g[p // 16, 8 * d + 4 * (p % 16):8 * d + 4 * (p % 16) + 4]) for p in range(16 * len(g))]


def special_rows(M, cols, d, seed, dt):
    """Rows with what a quantiser can go wrong at, head by head."""
    rng = np.random.default_rng(seed)
    x = of_bits(to_bits(rng.standard_normal((M, cols)), dt), dt).copy().reshape(-1, d)
    big = 65504.0 if dt == "fp16" else 3.3895313892515355e38
    kinds = [lambda v: v * 0, lambda v: v * 0 - 0.0, lambda v: v * 0 + 3.25, lambda v: np.where(np.arange(d) == 5, np.inf, v), lambda v: np.where(np.arange(d) == d - 1, np.nan, v),
             lambda v: np.where(np.arange(d) == 0, -np.inf, v), lambda v: np.where(v > 0, big, -big), lambda v: np.where(v > 0, big, 0), lambda v: v * 2.0**-22,
             lambda v: np.where(v > 0, 2.0**-24, 0), lambda v: rng.integers(0, 31, d) / 2, lambda v: rng.integers(0, 31, d) / 2 - 7.5, lambda v: v + 300, lambda v: v * 1000,
             lambda v: np.where(v > 1, big, v), lambda v: np.where(np.arange(d) == 3, 7e-5, 0), lambda v: v * 2.0**-90, lambda v: v * 2.0**-124, lambda v: v * 2.0**90]
    for i in range(len(x)):
        if i % 3 == 0:
            x[i] = kinds[i // 3 % len(kinds)](x[i])
    with np.errstate(over="ignore"):
        return of_bits(to_bits(x, dt), dt).reshape(M, cols)


CELL_SHAPES = [(1, 1, 64, 16, 1), (4, 2, 128, 16, 7), (12, 12, 64, 64, 33), (7, 7, 128, 256, 5), (10, 2, 64, 32, 200), (16, 8, 128, 128, 61)]


def bits_of(t):
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def from_bits(b, dt):
    import torch
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).cuda().view(dtype_of(dt))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("H,KV,d,P,M", CELL_SHAPES)
def test_append_and_load_bit_exact(H, KV, d, P, M, dt):
    import torch
    n_pages, cols = M // P + 5, (H + 2 * KV) * d
    x = special_rows(M, cols, d, M + d, dt)
    qkv = from_bits(to_bits(x, dt), dt).view(M, cols)
    size = lpq.lpq_cell_page_bytes(P, d)
    rng = np.random.default_rng(M)
    k, v = (rng.integers(0, 256, (n_pages, KV, size), dtype=np.uint8) for _ in range(2))
    kd, vd = torch.from_numpy(k.copy()).cuda(), torch.from_numpy(v.copy()).cuda()
    slots = random.Random(M).sample(range(n_pages * P), M)
    for bad, at in ((-1, 0), (n_pages * P, 2), (2**31 - 1, 4), (-2**31, 6)):
        if at < M and M > 1:
            slots[at] = bad
    values = np.full((M, cols), 77.0, np.float32)
    for row, s in enumerate(slots):
        if not 0 <= s < n_pages * P:
            continue
        for i, pages in enumerate((k, v)):
            for h in range(KV):
                at = (H + i * KV + h) * d
                codes, scale, zero = quantise(x[row, at:at + d], dt)
                cells, param = head_of(pages, s // P, h, d)[s % P]
                cells[:], param[:] = cell_bytes(codes, scale, zero)
                sf, zf = of_bits(scale, dt), of_bits(zero, dt)
                exact = sf.astype(np.float64) * codes + zf
                values[row, at:at + d] = exact.astype(np.float16) if dt == "fp16" else of_bits(to_bits((sf * codes).astype(np.float32) + zf, dt), dt)
    lpq.lpq_paged_append4(qkv, kd, vd, ints(slots))
    assert np.array_equal(kd.cpu().numpy(), k) and np.array_equal(vd.cpu().numpy(), v)
    out = torch.full((M, cols), 77.0, dtype=qkv.dtype, device="cuda")
    assert lpq.lpq_paged_load4(kd, vd, ints(slots), out) is out
    got = of_bits(bits_of(out), dt)
    assert np.array_equal(np.isnan(got), np.isnan(values))
    assert np.array_equal(np.nan_to_num(got, nan=1.0), np.nan_to_num(values, nan=1.0))
    # the same slot for several rows
    if M >= 5 and n_pages * P > slots[1] >= 0:
        again = torch.zeros_like(out)
        lpq.lpq_paged_load4(kd, vd, ints([slots[1]] * M), again)
        assert torch.equal(again[:, H * d:].contiguous().view(torch.int16), out[1:2, H * d:].expand(M, -1).contiguous().view(torch.int16))


# ---- norms and rotation ------------------------------------------------------------------------------------------------

def rotary_table(max_pos, rd, seed=0):
    import torch
    i = torch.arange(rd // 2, device="cuda", dtype=torch.float64)
    a = torch.arange(max_pos, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-i / (rd / 2))
    return torch.cat([a.cos(), a.sin()], 1).float()


def rotary_ref(x, H, KV, d, positions, table, interleaved, qg, kg, eps):
    """x [M][cols] -> (result, error of the 32-bit arithmetic) in 64 bits.  The sum of squares has d + 2 roundings, of 2^-24 each in units of itself, the root halves
    it, root, quotient and products five more; a rotation two products and a sum of |a cos| + |b sin|."""
    import torch
    M = x.shape[0]
    v = x.double().view(M, H + 2 * KV, d).clone()
    rel = torch.zeros((1, H + 2 * KV, 1), dtype=torch.float64, device="cuda")
    for h0, h1, g in ((0, H, qg), (H, H + KV, kg)):
        if g is not None:
            v[:, h0:h1] *= g.double() / torch.sqrt((v[:, h0:h1] ** 2).mean(2, keepdim=True) + eps)
            rel[:, h0:h1] = (0.5 * (d + 2) + 6) * 2.0**-24
    err = v.abs() * rel
    if table is not None:
        rd = table.shape[1]
        cos, sin = (t.double()[:, None, :] for t in table[positions.long()].chunk(2, 1))
        at = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
        qk = v[:, :H + KV]
        a, b = qk[..., at[0]].clone(), qk[..., at[1]].clone()
        ea, eb = err[:, :H + KV][..., at[0]].clone(), err[:, :H + KV][..., at[1]].clone()
        qk[..., at[0]], qk[..., at[1]] = a * cos - b * sin, b * cos + a * sin
        err[:, :H + KV][..., at[0]] = ea * cos.abs() + eb * sin.abs() + 3 * 2.0**-24 * ((a * cos).abs() + (b * sin).abs())
        err[:, :H + KV][..., at[1]] = eb * cos.abs() + ea * sin.abs() + 3 * 2.0**-24 * ((b * cos).abs() + (a * sin).abs())
    return v.view(M, -1), err.view(M, -1)


def check_rotary(H, KV, d, M, dt, rd, interleaved, norm, in_place, max_pos=300, seed=0):
    import torch
    g = gen(seed + M + rd)
    x = torch.randn((M, (H + 2 * KV) * d), generator=g, device="cuda").to(dtype_of(dt))
    if M > 3:
        x[3] = 0
    qg, kg = ((1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(x.dtype) if n else None for n in norm)
    r = random.Random(M)
    pos = [r.choice((0, 1, max_pos - 1, r.randrange(max_pos))) for _ in range(M)]
    slots = [r.randrange(1000) for _ in range(M)]
    skipped = []
    if M > 8:
        slots[1], slots[5], pos[2], pos[7] = -1, -2**31, -1, max_pos
        skipped = [1, 5] + ([2, 7] if rd else [])
    table = rotary_table(max_pos, rd) if rd else None
    keep = [i for i in range(M) if i not in skipped]
    ref, err = rotary_ref(x[keep], H, KV, d, ints([pos[i] for i in keep]), table, interleaved, qg, kg, 1e-5)
    before = x.clone()
    out = x if in_place else torch.full_like(x, 77.0)
    got = lpq.lpq_qk_norm_rotary(x, ints(pos), H, KV, cos_sin=table, interleaved=interleaved, q_gamma=qg, k_gamma=kg, eps=1e-5, slots=ints(slots), out=None if in_place else out)
    assert got is out
    u = {"fp16": 2.0**-11, "bf16": 2.0**-8}[dt]
    tol = u * (ref.abs() + err) + err + 2.0**-25
    far = (out[keep].double() - ref).abs() / tol
    assert float(far.max()) <= 1.0, float(far.max())
    assert torch.equal(out[keep][:, (H + KV) * d:], before[keep][:, (H + KV) * d:]), "V"
    for i in skipped:
        assert torch.equal(out[i], before[i] if in_place else torch.full_like(before[i], 77.0)), "row %d is to be left" % i
    if not in_place:
        assert torch.equal(x, before)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "adjacent"])
@pytest.mark.parametrize("H,KV,d,M,rd,norm,in_place", [
    (1, 1, 64, 1, 64, (1, 1), True), (4, 2, 128, 9, 128, (1, 1), False), (12, 12, 64, 33, 32, (0, 0), True), (40, 40, 128, 21, 128, (0, 0), False), (64, 8, 128, 50, 64, (1, 1), True),
    (7, 7, 128, 11, 16, (1, 0), True), (7, 1, 64, 300, 48, (0, 1), False), (16, 2, 64, 10, 0, (1, 1), True), (9, 3, 128, 12, 112, (0, 0), True), (72, 8, 128, 400, 96, (1, 1), False),
    (3, 1, 128, 10, 0, (0, 0), False),
])
def test_norm_and_rotation(H, KV, d, M, rd, norm, in_place, interleaved, dt):
    check_rotary(H, KV, d, M, dt, rd, interleaved, norm, in_place)


def test_rotation_without_slots_and_far_positions():
    """No slots: every row; a table of 100000 positions; infinities and NaN stay in their pair without norms, in their head with."""
    import torch
    H, KV, d, M = 4, 2, 64, 40
    x = torch.randn((M, (H + 2 * KV) * d), generator=gen(4), device="cuda").half()
    table = rotary_table(100000, d)
    pos = ints([99999 - 7 * i for i in range(M)])
    ref, err = rotary_ref(x, H, KV, d, pos, table, False, None, None, 1e-5)
    y = lpq.lpq_qk_norm_rotary(x, pos, H, KV, cos_sin=table, out=torch.empty_like(x))
    assert float(((y.double() - ref).abs() / (2.0**-11 * (ref.abs() + err) + err + 2.0**-25)).max()) <= 1.0
    bad = x.clone()
    bad[0, 3], bad[1, d + 40] = math.inf, math.nan
    z = lpq.lpq_qk_norm_rotary(bad, pos, H, KV, cos_sin=table, out=torch.empty_like(x))
    odd = (~torch.isfinite(z)).nonzero().tolist()
    assert odd == [[0, 3], [0, 35], [1, d + 8], [1, d + 40]]
    same = torch.ones_like(z, dtype=torch.bool)
    for i, j in odd:
        same[i, j] = False
    assert torch.equal(z[same], y[same])


# ---- attention ----------------------------------------------------------------------------------------------------------

def attention_ref(q, cells, ok, pos, slopes, tile, dt):
    """q [T][H][d]; cells: codes [2][L][KV][d], scale and zero [2][L][KV] in 64 bits (K, V); ok [L], pos [T].  -> (out, bound without the output's rounding)."""
    import torch
    T, H, d = q.shape
    codes, scale, zero = cells
    L, KV = codes.shape[1], codes.shape[2]
    out, E = (torch.zeros((T, H, d), dtype=torch.float64, device="cuda") for _ in range(2))
    if L == 0:
        return out, E
    j = torch.arange(L, device="cuda")
    vis = ok[None, :] & (j[None, :] <= pos[:, None])
    dist = (j[None, :] - pos[:, None]).double()
    lg, none = math.log2(math.e), torch.zeros((), dtype=torch.float64, device="cuda")
    fin = lambda x: torch.where(torch.isfinite(x), x, none)
    for h in range(H):
        g = h // (H // KV)
        sk, zk, sv, zv = (fin(t[i, :, g]) * ok for i in (0, 1) for t in (scale, zero))
        ck, cv = codes[0, :, g].double() * ok[:, None], codes[1, :, g].double() * ok[:, None]
        kh, vh = ck * sk[:, None] + zk[:, None], cv * sv[:, None] + zv[:, None]
        qh = q[:, h].double()
        s = (qh @ kh.t().contiguous()) / math.sqrt(d)
        size = qh.abs().sum(1, keepdim=True) / math.sqrt(d)                      # sum |q_i|
        err = (d + 8) * 2.0**-24 * size * (15 * sk + zk.abs())[None, :]
        if tile:
            err = err + U16 * (qh.abs() @ kh.abs().t().contiguous()) / math.sqrt(d) + 2.0**-24 * size * torch.maximum(15 * sk, zk.abs()).amax()
        else:
            err = err + 2.0**-18 * size * sk[None, :]
        if slopes is not None:
            s = s + float(slopes[h]) * dist
            err = err + 2.0**-24 * (float(slopes[h]) * dist).abs()
        s = torch.where(vis, s, torch.full_like(s, -math.inf))
        top = s.amax(1, keepdim=True)
        w = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total > 0, total, torch.ones_like(total))
        o = w @ vh
        odd = ~(torch.isfinite(scale[:, :, g]) & torch.isfinite(zero[:, :, g])).all(0)
        o[(vis & odd[None, :]).any(1)] = math.nan                                # a position stored as NaN
        out[:, h] = o
        A, n = w @ vh.abs(), L
        arg = err * lg + 3 * 2.0**-24 * (fin(s).abs() + fin(top).abs()) * lg
        e = 2 * (math.log(2) * torch.where(vis, arg, none).amax(1, keepdim=True) + 2.0**-22) * A + 2 * n * 2.0**-24 * (w @ (15 * sv + zv.abs()))[:, None]
        if tile:
            e = e + U16 * A + 2.0**-24 * torch.maximum(15 * sv, zv.abs()).amax() + U16 * (A + fin(o).abs()) + n * 2.0**-25 * vh.abs().amax()
        else:
            e = e + (2.0**-18 * (w @ sv) + 8 * n * 2.0**-33 * (w * sv[None, :]).amax(1))[:, None] + U16 * (w @ (sv[:, None] * (cv - 8).abs()))
        E[:, h] = e
    return out, E


def check_attention(got, parts, what=""):
    """parts: [(rows, reference)]; rows that no part names have to be as they were: 77."""
    import torch
    u = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}[got.dtype]
    left = torch.ones(got.shape[0], dtype=torch.bool, device="cuda")
    for (r0, r1), (out, E) in parts:
        left[r0:r1] = False
        if r1 == r0:
            continue
        g = got[r0:r1].double().view(out.shape)
        nan = torch.isnan(out)
        assert torch.equal(torch.isnan(g), nan), what + ": NaN at other places"
        far = torch.where(nan, torch.zeros_like(out), (g - out).abs() / (u * (out.abs() + E) + E + 2.0**-25))
        assert float(far.max()) <= 1.0, "%s: rows %d..%d, %.2f of the bound at %s" % (what, r0, r1, float(far.max()), np.unravel_index(int(far.argmax()), far.shape))
    assert bool((got[left] == 77).all()), what + ": rows behind the last sequence"


class Cells:
    """A pool of random cells (stale ones everywhere), sequences (cached positions, new tokens) on pages in random order."""

    def __init__(self, seqs, H, KV, d, P, dt, pad=0, seed=0, spare=3, width_extra=1, spread=0.0):
        import torch
        self.seqs, self.H, self.KV, self.d, self.P, self.dt = seqs, H, KV, d, P, dt
        g = gen(seed + 17 * len(seqs) + H + P)
        have = [-(-(p + q) // P) for p, q in seqs]
        self.n_pages = sum(have) + spare
        ids = torch.randperm(self.n_pages, generator=g, device="cuda").tolist()
        width = max(have) + width_extra
        self.table, at = [], 0
        for n in have:
            self.table.append(ids[at:at + n] + [-1] * (width - n))
            at += n
        self.cu = np.concatenate([[0], np.cumsum([q for _, q in seqs])])
        self.M = max(1, int(self.cu[-1]) + pad)
        qkv = torch.randn((self.M, (H + 2 * KV) * d), generator=g, device="cuda")
        qkv[:, :H * d] *= 2
        self.qkv = qkv.to(dtype_of(dt))
        # scales around 1/3, of `spread` binades more either way; zeros near -7.5 of them
        shape = (2, self.n_pages, KV, P)
        scale = 0.2 + 0.25 * torch.rand(shape, generator=g, device="cuda")
        if spread:
            scale *= torch.exp2(spread * (2 * torch.rand(shape, generator=g, device="cuda") - 1))
        zero = scale * (-7.5 + torch.randn(shape, generator=g, device="cuda"))
        self.param = torch.stack([scale, zero], -1).to(dtype_of(dt))
        self.codes = torch.randint(0, 16, (*shape, d), generator=g, device="cuda", dtype=torch.uint8)
        self.write()

    def write(self):
        """The pages' bytes from self.codes and self.param."""
        import torch
        n, KV, P, d = self.n_pages, self.KV, self.P, self.d
        c = self.codes.view(2, n, KV, P // 16, 16, d // 8, 8).int()
        word = sum(c[..., e] << (4 * (e // 2) + 16 * (e % 2)) for e in range(8))
        cells = word.contiguous().view(torch.uint8).view(2, n, KV, P // 16, 8 * d)
        param = self.param.contiguous().view(torch.uint8).view(2, n, KV, P // 16, 64)
        self.k, self.v = torch.cat([cells, param], -1).view(2, n, KV, P * (d // 2 + 4)).unbind(0)
        assert self.k.shape[2] == lpq.lpq_cell_page_bytes(P, d)

    def run(self, alibi=False, max_q=None, max_kv=None, kv_lens=None, out=None, loose=False, **how):
        import torch
        kv = [p + q for p, q in self.seqs] if kv_lens is None else kv_lens
        out = torch.full((self.M, self.H * self.d), 77.0, dtype=self.qkv.dtype, device="cuda") if out is None else out
        slopes = slopes_of(self.H, alibi)
        lpq.lpq_paged_attention4(self.qkv, self.k, self.v, ints(self.table), ints(self.cu), ints(kv), max_q=max_q, max_kv=max_kv, alibi_slopes=slopes, out=out, **how)
        return out, self.parts(kv, slopes, loose)

    def parts(self, kv, slopes, loose=False):
        import torch
        res = []
        for s, (past, q) in enumerate(self.seqs):
            L = min(max(kv[s], 0), len(self.table[s]) * self.P)
            ids = torch.tensor([self.table[s][j // self.P] for j in range(L)], dtype=torch.long, device="cuda")
            ok = (ids >= 0) & (ids < self.n_pages)
            at, off = torch.where(ok, ids, torch.zeros_like(ids)), torch.arange(L, device="cuda") % self.P
            codes, param = self.codes[:, at, :, off].transpose(0, 1), self.param[:, at, :, off].transpose(0, 1).double()
            param = torch.where(ok[None, :, None, None], param, torch.zeros_like(param))
            r0, r1 = self.cu[s], self.cu[s + 1]
            pos = max(kv[s], 0) - q + torch.arange(q, device="cuda")
            tile = loose or q * (self.H // self.KV) > 32
            res.append(((r0, r1), attention_ref(self.qkv[r0:r1, :self.H * self.d].view(q, self.H, self.d), (codes, param[..., 0], param[..., 1]), ok, pos, slopes, tile, self.dt)))
        return res


def longest(seqs):
    return dict(max_q=max(q for _, q in seqs), max_kv=max(a + b for a, b in seqs))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("alibi", [False, True], ids=["plain", "alibi"])
@pytest.mark.parametrize("seqs,H,KV,d,P,pad", [
    ([(0, 1)], 1, 1, 64, 16, 0), ([(0, 1), (15, 1), (16, 1), (17, 1)], 4, 2, 128, 16, 3), ([(31, 1), (32, 1), (127, 1), (128, 1), (700, 1)], 5, 5, 64, 32, 0),
    ([(1000, 1)], 12, 12, 128, 64, 0), ([(3000, 1), (2, 1)], 8, 1, 128, 256, 1), ([(450, 1)] * 9, 32, 2, 64, 64, 0), ([(777, 1), (1290, 1)], 14, 2, 128, 128, 2),
    ([(5000, 1)], 40, 2, 64, 16, 0), ([(600, 1), (60, 1)], 34, 1, 128, 32, 0), ([(333, 1)], 80, 2, 128, 64, 0),
], ids=lambda v: "_".join("%d+%d" % x for x in v[:4]) if isinstance(v, list) else str(v))
def test_decode(seqs, H, KV, d, P, pad, alibi, dt):
    check_attention(*Cells(seqs, H, KV, d, P, dt, pad).run(alibi, max_q=1), what="decode")


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("alibi", [False, True], ids=["plain", "alibi"])
@pytest.mark.parametrize("seqs,H,KV,d,P,pad", [
    ([(0, 5)], 1, 1, 64, 16, 0), ([(100, 3), (9, 2), (0, 4)], 8, 2, 128, 16, 2), ([(900, 8), (30, 1)], 4, 1, 64, 64, 0), ([(40, 16), (0, 1), (7, 0)], 2, 2, 128, 32, 0),
    ([(64, 64)], 2, 2, 64, 64, 0), ([(0, 130), (250, 33)], 6, 2, 128, 256, 7), ([(1500, 100)], 16, 2, 128, 128, 0), ([(2000, 40), (100, 200)], 4, 4, 64, 16, 1),
    ([(3000, 20)], 7, 1, 128, 64, 0), ([(500, 1), (700, 90), (3, 1), (0, 1), (90, 31)], 8, 4, 64, 16, 5), ([(10, 1), (900, 300), (1200, 1)], 34, 1, 64, 32, 2),
    ([(200, 1), (2100, 300)], 56, 8, 128, 32, 3),
], ids=lambda v: "_".join("%d+%d" % x for x in v[:4]) if isinstance(v, list) else str(v))
def test_chunks_and_mixed(seqs, H, KV, d, P, pad, alibi, dt):
    """Chunks short and long, alone and beside sequences that decode: the streaming kernel's one and two column tiles, the tile kernel, its splits, and both."""
    check_attention(*Cells(seqs, H, KV, d, P, dt, pad).run(alibi, **longest(seqs)), what="chunks")
