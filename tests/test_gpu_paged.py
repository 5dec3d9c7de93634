"""GPU parity of the operators over paged caches and packed rows: the plan (integers, equal), the append (bit-exact) and both attentions against
plain 64-bit implementations, at the sizes, layouts and masks where they can go wrong, and a run of them together.

Tolerance of an attention output, element by element.  With weights w_j (summing to 1), A = sum w_j |v_j| and u half a step of the output's type
(2^-11 fp16, 2^-8 bf16):
  * the weights are rounded to that type, in the products and in the sum that divides them: w_j (1 + d_j) with |d_j| <= u gives
    sum w_j (1 + d_j) v_j / sum w_j (1 + d_j) = (out + sum w_j d_j v_j) / (1 + sum w_j d_j), off by                             u A + u |out|
    to first order; a weight below fp16's normal range by half its smallest step instead, beside a sum of at least 1:       n 2^-25 max |v|
  * a weight exp2(s) has the error of its exponent: the score is a 32-bit sum of D products of 16-bit numbers ((D + 4) 2^-24 sum |q_i k_i|),
    scaled, biased and shifted by the row's maximum in 32 bits (3 roundings of at most 2^-24 (|s| + |max|)), and exp2 itself 2^-22;
    the error counts for the weight and for the sum it is divided by:                     2 (ln 2 * that + 2^-22) A
  * 32-bit sums over n keys, of the products and of the weights:                          2 n 2^-24 A
  * the output's own rounding, u |out|, and half the smallest step where it is subnormal (fp16: 2^-25)."""
import math
import random

import numpy as np
import pytest

import paper_2403_01136_amd as lpq

pytestmark = pytest.mark.gpu
DTYPES = {"fp16": 0, "bf16": 1}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU (no fallback path)"
    lpq.load_library()


def dtype_of(name):
    import torch
    return {"fp16": torch.float16, "bf16": torch.bfloat16}[name]


def ints(values):
    import torch
    return torch.tensor(np.asarray(values), dtype=torch.int32, device="cuda")


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


# ---- the plan ---------------------------------------------------------------------------------------------------------

def plan_ref(past, q_lens, table, ring, head, free, P, M):
    """The step one sequence, page and token after the other."""
    n_pages, width = len(ring), len(table[0])
    table, ring = [list(t) for t in table], list(ring)
    supply = [ring[(head + i) % n_pages] for i in range(free)]
    cu, kv, slots, pos = [0], [], [-1] * M, [0] * M
    rows = wanted = taken = starved = 0
    back = []
    for s, (p, q) in enumerate(zip(past, q_lens)):
        p = max(p, 0)
        if q < 0:
            back += table[s][:min(-(-p // P), width)]
            cu.append(min(rows, M)), kv.append(0)
            continue
        start, rows = rows, rows + q
        cu.append(min(rows, M))
        ok = q == 0 or (rows <= M and p + q <= width * P)
        if ok and q:
            held, need = -(-p // P), -(-(p + q) // P) - -(-p // P)
            wanted += need
            ok = need == 0 or wanted <= free
            if ok:
                if need:
                    table[s][held:held + need] = supply[wanted - need:wanted]
                    taken = wanted
                for t in range(q):
                    page = table[s][(p + t) // P]
                    pos[start + t] = p + t
                    slots[start + t] = page * P + (p + t) % P if 0 <= page < n_pages else -1
        starved += not ok
        kv.append(p + q if ok else p)
    back = back[:n_pages - free]
    for i, page in enumerate(back):
        ring[(head + free + i) % n_pages] = page
    return dict(cu_q=cu, kv_lens=kv, slots=slots, positions=pos, counters=[(head + taken) % n_pages, free - taken + len(back)],
                info=[cu[-1], taken, len(back), starved], table=table, ring=ring)


def plan_case(seed, n, P, q_of, past_hi, spare, width_extra=2, pad=3):
    """(past, q_lens, table, ring, head, free, M): sequences that hold the pages of their positions, the rest on the ring from a random place on."""
    r = random.Random(seed)
    past = [r.choice((0, 1, P - 1, P, r.randint(0, past_hi))) for _ in range(n)]
    q = [q_of(r) for _ in range(n)]
    held = [-(-p // P) for p in past]
    need = [-(-(p + max(x, 0)) // P) - h for p, x, h in zip(past, q, held)]
    free = max(0, sum(need) + spare)
    n_pages = sum(held) + free + r.randint(0, 3) or 1
    ids = list(range(n_pages))
    r.shuffle(ids)
    width = max(h + e for h, e in zip(held, need)) + width_extra
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-7] * (width - h))
        at += h
    head = r.randrange(n_pages)
    ring = [-9] * n_pages
    for i in range(free):
        ring[(head + i) % n_pages] = ids[at + i]
    return past, q, table, ring, head, free, max(1, sum(max(x, 0) for x in q) + pad)


def run_plan(past, q, table, ring, head, free, P, M, in_place=False):
    import torch
    past_d, q_d, table_d, ring_d, counters = ints(past), ints(q), ints(table), ints(ring), ints([head, free])
    n = len(past)
    plan = tuple(torch.full((m,), -123, dtype=torch.int32, device="cuda") for m in (n + 1, n, M, M, 2, 4))
    if in_place:
        plan = (plan[0], past_d, plan[2], plan[3], counters, plan[5])
    got = lpq.lpq_paged_plan(past_d, q_d, table_d, ring_d, counters, P, M, plan=plan)
    out = {k: getattr(got, k).tolist() for k in got._fields}
    out.update(table=table_d.tolist(), ring=ring_d.tolist())
    return out


def check_plan(case, P, **k):
    want = plan_ref(*case[:6], P, case[6])
    got = run_plan(*case[:6], P, case[6], **k)
    for name, w in want.items():
        assert got[name] == w, name
    return want


DECODE, MIXED = (lambda r: 1), (lambda r: r.choice((1, 1, 1, 0, -1, r.randint(2, 90))))


@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "in_place"])
@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("n", [1, 2, 7, 64, 65, 129, 300, 2048])
def test_plan(n, P, in_place):
    for i, q_of in enumerate((DECODE, MIXED)):
        check_plan(plan_case(100 * n + P + i, n, P, q_of, 700, 5), P, in_place=in_place)


@pytest.mark.parametrize("n,lo,hi", [(3, 1500, 2500), (24, 100, 900), (200, 0, 60), (1, 9000, 9000)])
def test_plan_many_rows(n, lo, hi):
    """More rows than one launch takes: the second launch's path."""
    case = plan_case(n, n, 32, lambda r: r.choice((r.randint(lo, hi), r.randint(lo, hi), -1 if n > 3 else hi)), 400, 9)
    check_plan(case, 32)
    check_plan(case, 32, in_place=True)


@pytest.mark.parametrize("n", [2, 30, 600, 2048])
def test_plan_many_rows_starved(n):
    """The same without the pages, the rows or the table entries that all of them would need; rows near the line between one launch and two."""
    for rows in (6144, 6145, 12000):
        case = plan_case(n + rows, n, 16, lambda r: r.choice((0, -1, r.randint(0, 2 * rows // n + 1), 2 * rows // n)), 90, 0)
        past, q, table, ring, head, free, M = case
        for f, m in ((free, rows), (free // 2, rows + 900), (0, rows), (max(free - 1, 0), M)):
            check_plan((past, q, table, ring, head, f, m), 16, in_place=f == free // 2)
        check_plan((past, q, [t[:max(1, len(t) - 3)] for t in table], ring, head, free, rows), 16)


@pytest.mark.parametrize("n", [5, 40, 257])
def test_plan_starved(n):
    """Too few pages, rows behind the batch, positions behind the table, an empty pool; finished sequences return theirs all the same."""
    case = plan_case(n, n, 16, MIXED, 300, 0)
    past, q, table, ring, head, free, M = case
    for f in (0, 1, free // 2, max(free - 1, 0)):
        assert check_plan((past, q, table, ring, head, f, M), 16)["info"][1] <= f
    rows = sum(max(x, 0) for x in q)
    for m in (1, rows // 2, max(rows - 1, 1)):
        check_plan((past, q, table, ring, head, free, m), 16)
    narrow = [t[:max(1, len(t) - 3)] for t in table]
    check_plan((past, q, narrow, ring, head, free, M), 16)
    check_plan((past, [-1] * n, table, ring, head, free, M), 16)            # everybody has finished
    check_plan((past, [0] * n, table, ring, head, free, M), 16)             # nobody has anything


def test_plan_odd_integers():
    """Lengths at the ends of their type, counters out of range, tables with ids that are no pages: defined results, nothing out of place."""
    big = 2**31 - 1
    past, q, table = [big, 5, -4, big, 20, 33], [1, big, 3, -1, 2, 0], [[-1, 90, 4]] * 6
    want = plan_ref([big, 5, 0, big, 20, 33], q, table, list(range(10)), 3, 4, 16, 50)
    got = run_plan(past, q, table, list(range(10)), 3, 4, 16, 50)
    for name in want:
        assert got[name] == want[name], name
    for head, free, h, f in ((-5, 3, 0, 3), (23, 3, 3, 3), (2, -1, 2, 0), (2, 99, 2, 10)):
        want = plan_ref([0, 17], [1, 20], [[-1] * 4] * 2, list(range(10)), h, f, 16, 30)
        got = run_plan([0, 17], [1, 20], [[-1] * 4] * 2, list(range(10)), head, free, 16, 30)
        for name in want:
            assert got[name] == want[name], name


def test_plan_positions_of_rows_without_a_slot():
    """A served row has its position also where its table entry is no page of the pool (slot -1); a starved one and one of nobody have 0."""
    got = run_plan([20, 5, 40], [2, 30, 1], [[3, -1, -1], [9, -1, -1], [0, 1, 99]], [4, 5, 6, 7, 8, 2, -9, -9, -9, -9], 0, 1, 16, 35)
    assert got["slots"][:2] == [-1, -1] and got["positions"][:2] == [20, 21]        # entry 1 of the first sequence is no page
    assert got["slots"][2:32] == [-1] * 30 and got["positions"][2:32] == [0] * 30   # two pages wanted, one free
    assert got["slots"][32] == -1 and got["positions"][32] == 40                    # page 99 of a pool of 10
    assert got["slots"][33:] == [-1, -1] and got["positions"][33:] == [0, 0] and got["info"][3] == 1


# ---- the append -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("H,KV,d,P,M", [(1, 1, 64, 16, 1), (4, 2, 128, 16, 7), (12, 12, 64, 64, 33), (7, 7, 128, 256, 5), (10, 2, 64, 32, 300), (64, 8, 128, 128, 129)])
def test_append_bit_exact(H, KV, d, P, M, dt):
    import torch
    n_pages = M // P + 5
    g = gen(M + d)
    qkv = torch.randn((M, (H + 2 * KV) * d), generator=g, device="cuda").to(dtype_of(dt))
    k, v = (torch.randn((n_pages, KV, P, d), generator=g, device="cuda").to(dtype_of(dt)) for _ in range(2))
    r = random.Random(M)
    slots = r.sample(range(n_pages * P), M)
    for bad, at in ((-1, 0), (n_pages * P, 2), (2**31 - 1, 4), (-2**31, 6)):
        if at < M and M > 1:
            slots[at] = bad
    k_ref, v_ref = k.clone(), v.clone()
    for row, s in enumerate(slots):
        if 0 <= s < n_pages * P:
            new = qkv[row, H * d:].view(2, KV, d)
            k_ref[s // P, :, s % P], v_ref[s // P, :, s % P] = new[0], new[1]
    lpq.lpq_paged_append(qkv, k, v, ints(slots))
    assert torch.equal(k.view(torch.int16), k_ref.view(torch.int16)) and torch.equal(v.view(torch.int16), v_ref.view(torch.int16))


# ---- attention --------------------------------------------------------------------------------------------------------

def attention_ref(q, k, v, ok, pos, slopes):
    """q [T][H][d], k, v [L][KV][d] (any values where ok is false), ok [L], pos [T] -> (out [T][H][d], A, bound without the output's rounding and the weights'
    relative one) in 64 bits; per head."""
    import torch
    T, H, d = q.shape
    L, KV = k.shape[0], k.shape[1]
    out, A, E = (torch.zeros((T, H, d), dtype=torch.float64, device="cuda") for _ in range(3))
    if L == 0:
        return out, A, E
    j = torch.arange(L, device="cuda")
    vis = ok[None, :] & (j[None, :] <= pos[:, None])
    dist = (j[None, :] - pos[:, None]).double()
    for h in range(H):
        kh, vh = k[:, h // (H // KV)].double(), v[:, h // (H // KV)].double()
        kh = torch.where(ok[:, None], kh, torch.zeros_like(kh))
        qh = q[:, h].double()
        s = (qh @ kh.t().contiguous()) / math.sqrt(d)
        mag = (qh.abs() @ kh.abs().t().contiguous()) / math.sqrt(d)
        if slopes is not None:
            s = s + float(slopes[h]) * dist
            mag = mag + (float(slopes[h]) * dist).abs()
        s = torch.where(vis, s, torch.full_like(s, -math.inf))
        top = s.amax(1, keepdim=True)
        w = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total > 0, total, torch.ones_like(total))
        # values that a row may not see have weight zero, whatever they are: 0 * inf is left out
        vz = torch.where(torch.isfinite(vh), vh, torch.zeros_like(vh))
        o = w @ vz
        odd = (~torch.isfinite(vh)).any(1)
        if bool(odd.any()):
            seen = (vis & odd[None, :]).any(1)
            o[seen] = (w[seen][:, :, None] * vh[None]).sum(1) if int(seen.sum()) * L * d < 2e8 else math.nan
        out[:, h] = o
        A[:, h] = w @ vz.abs()
        lg = math.log2(math.e)
        fin = lambda x: torch.where(torch.isfinite(x), x, torch.zeros_like(x))
        arg = ((d + 4) * mag * lg + 3 * (fin(s).abs() * lg + fin(top).abs() * lg)) * 2.0**-24
        E[:, h] = (w * (2 * (math.log(2) * torch.where(vis, arg, torch.zeros_like(arg)).amax(1, keepdim=True) + 2.0**-22) + 2 * L * 2.0**-24)) @ vz.abs()
        if q.dtype == torch.float16:
            E[:, h] += L * 2.0**-25 * vz.abs().amax()
    return out, A, E


def check_attention(got, parts, what=""):
    """parts: [(rows, reference)]; rows that no part names have to be as they were: 77."""
    import torch
    u = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}[got.dtype]
    left = torch.ones(got.shape[0], dtype=torch.bool, device="cuda")
    for (r0, r1), (out, A, E) in parts:
        left[r0:r1] = False
        if r1 == r0:
            continue
        g = got[r0:r1].double().view(out.shape)
        nan = torch.isnan(out)
        assert torch.equal(torch.isnan(g), nan), what + ": NaN at other places"
        tol = u * (A + out.abs()) + E + u * (out.abs() + u * A + E) + 2.0**-25
        far = torch.where(nan, torch.zeros_like(out), (g - out).abs() / tol)
        assert float(far.max()) <= 1.0, "%s: rows %d..%d, %.2f of the bound at %s" % (what, r0, r1, float(far.max()), np.unravel_index(int(far.argmax()), far.shape))
    assert bool((got[left] == 77).all()), what + ": rows behind the last sequence"


def slopes_of(H, alibi):
    import torch
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / H) for i in range(H)], dtype=torch.float32, device="cuda") if alibi else None


def packed_run(lens, H, KV, d, dt, alibi, pad=0, seed=0, max_q=None, edit=None):
    import torch
    M = max(1, sum(lens) + pad)
    qkv = torch.randn((M, (H + 2 * KV) * d), generator=gen(seed + M + H), device="cuda")
    qkv[:, :H * d] *= 2
    qkv = qkv.to(dtype_of(dt))
    if edit:
        edit(qkv)
    cu = np.concatenate([[0], np.cumsum(lens)])
    out = torch.full((M, H * d), 77.0, dtype=qkv.dtype, device="cuda")
    slopes = slopes_of(H, alibi)
    lpq.lpq_packed_attention(qkv, ints(cu), H, KV, max_q=max_q, alibi_slopes=slopes, out=out)
    parts = []
    for s, n in enumerate(lens):
        rows = qkv[cu[s]:cu[s + 1]]
        q, k, v = rows[:, :H * d].view(n, H, d), rows[:, H * d:(H + KV) * d].view(n, KV, d), rows[:, (H + KV) * d:].view(n, KV, d)
        parts.append(((cu[s], cu[s + 1]), attention_ref(q, k, v, torch.ones(n, dtype=torch.bool, device="cuda"), torch.arange(n, device="cuda"), slopes)))
    return out, parts


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("alibi", [False, True], ids=["plain", "alibi"])
@pytest.mark.parametrize("lens,H,KV,d,pad", [
    ([1], 1, 1, 64, 0), ([1, 1, 1], 4, 2, 128, 2), ([64], 3, 3, 128, 0), ([63, 65, 0, 2], 6, 2, 64, 5), ([127, 128, 129], 4, 4, 64, 1), ([200, 1, 17, 0, 300], 12, 12, 64, 9),
    ([130, 33], 14, 2, 128, 0), ([5, 90], 40, 1, 64, 3), ([700], 2, 2, 128, 0), ([513, 31], 20, 4, 128, 40), ([16] * 70, 8, 8, 64, 0), ([300], 130, 1, 64, 0),
], ids=lambda v: "x".join(map(str, v[:5])) if isinstance(v, list) else str(v))
def test_packed_attention(lens, H, KV, d, pad, alibi, dt):
    check_attention(*packed_run(lens, H, KV, d, dt, alibi, pad), what="packed %s" % lens)


def test_packed_attention_long():
    """Longer than a tile's and a split's worth, with few rows elsewhere; a length expected that is not the longest."""
    check_attention(*packed_run([2300, 40], 4, 1, 128, "fp16", False), what="long")
    check_attention(*packed_run([1900, 40], 4, 1, 64, "bf16", True, max_q=8), what="long, unexpected")


@pytest.mark.parametrize("n", [64, 65, 100, 2048])
def test_packed_attention_many_sequences(n):
    r = random.Random(n)
    check_attention(*packed_run([r.choice((0, 1, 2, 9, 40)) if n < 2048 else r.choice((0, 1, 2)) for _ in range(n)], 4, 2, 64, "fp16", False, 3), what="many")


class Paged:
    """A pool filled with random values (stale ones everywhere), sequences (cached positions, new tokens) on pages in random order."""

    def __init__(self, seqs, H, KV, d, P, dt, pad=0, seed=0, spare=3, width_extra=1):
        import torch
        self.seqs, self.H, self.KV, self.d, self.P = seqs, H, KV, d, P
        g = gen(seed + 17 * len(seqs) + H + P)
        have = [-(-(p + q) // P) for p, q in seqs]
        self.n_pages = sum(have) + spare
        ids = torch.randperm(self.n_pages, generator=g, device="cuda").tolist()
        width = max(have) + width_extra
        self.table, at = [], 0
        for h in have:
            self.table.append(ids[at:at + h] + [-1] * (width - h))
            at += h
        self.cu = np.concatenate([[0], np.cumsum([q for _, q in seqs])])
        self.M = max(1, int(self.cu[-1]) + pad)
        qkv = torch.randn((self.M, (H + 2 * KV) * d), generator=g, device="cuda")
        qkv[:, :H * d] *= 2
        self.qkv = qkv.to(dtype_of(dt))
        self.k, self.v = (torch.randn((self.n_pages, KV, P, d), generator=g, device="cuda").to(dtype_of(dt)) for _ in range(2))

    def run(self, alibi=False, max_q=None, max_kv=None, kv_lens=None, out=None):
        import torch
        kv = [p + q for p, q in self.seqs] if kv_lens is None else kv_lens
        out = torch.full((self.M, self.H * self.d), 77.0, dtype=self.qkv.dtype, device="cuda") if out is None else out
        slopes = slopes_of(self.H, alibi)
        lpq.lpq_paged_attention(self.qkv, self.k, self.v, ints(self.table), ints(self.cu), ints(kv), max_q=max_q, max_kv=max_kv, alibi_slopes=slopes, out=out)
        return out, self.parts(kv, slopes)

    def parts(self, kv, slopes):
        import torch
        res = []
        for s, (past, q) in enumerate(self.seqs):
            L = min(max(kv[s], 0), len(self.table[s]) * self.P)
            ids = torch.tensor([self.table[s][j // self.P] for j in range(L)], dtype=torch.long, device="cuda")
            ok = (ids >= 0) & (ids < self.n_pages)
            off = torch.arange(L, device="cuda") % self.P
            k, v = (t[torch.where(ok, ids, torch.zeros_like(ids)), :, off] for t in (self.k, self.v))
            v = torch.where(ok[:, None, None], v, torch.zeros_like(v))
            r0, r1 = self.cu[s], self.cu[s + 1]
            pos = max(kv[s], 0) - q + torch.arange(q, device="cuda")
            res.append(((r0, r1), attention_ref(self.qkv[r0:r1, :self.H * self.d].view(q, self.H, self.d), k, v, ok, pos, slopes)))
        return res


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("alibi", [False, True], ids=["plain", "alibi"])
@pytest.mark.parametrize("seqs,H,KV,d,P,pad", [
    ([(0, 1)], 1, 1, 64, 16, 0), ([(0, 1), (15, 1), (16, 1), (17, 1)], 4, 2, 128, 16, 3), ([(31, 1), (32, 1), (127, 1), (128, 1), (700, 1)], 5, 5, 64, 32, 0),
    ([(1000, 1)], 12, 12, 128, 64, 0), ([(3000, 1), (2, 1)], 8, 1, 128, 256, 1), ([(450, 1)] * 9, 32, 2, 64, 64, 0), ([(777, 1), (1290, 1)], 14, 2, 128, 128, 2),
    ([(5000, 1)], 40, 2, 64, 16, 0), ([(600, 1), (60, 1)], 34, 1, 128, 32, 0), ([(333, 1)], 80, 2, 128, 64, 0),
], ids=lambda v: "_".join("%d+%d" % x for x in v[:4]) if isinstance(v, list) else str(v))
def test_paged_decode(seqs, H, KV, d, P, pad, alibi, dt):
    check_attention(*Paged(seqs, H, KV, d, P, dt, pad).run(alibi, max_q=1), what="decode")


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("alibi", [False, True], ids=["plain", "alibi"])
@pytest.mark.parametrize("seqs,H,KV,d,P,pad", [
    ([(0, 5)], 1, 1, 64, 16, 0), ([(100, 3), (9, 2), (0, 4)], 8, 2, 128, 16, 2), ([(900, 8), (30, 1)], 4, 1, 64, 64, 0), ([(40, 16), (0, 1), (7, 0)], 2, 2, 128, 32, 0),
    ([(64, 64)], 2, 2, 64, 64, 0), ([(0, 130), (250, 33)], 6, 2, 128, 256, 7), ([(1500, 100)], 16, 2, 128, 128, 0), ([(2000, 40), (100, 200)], 4, 4, 64, 16, 1),
    ([(3000, 20)], 7, 1, 128, 64, 0), ([(500, 1), (700, 90), (3, 1), (0, 1), (90, 31)], 8, 4, 64, 16, 5), ([(10, 1), (900, 300), (1200, 1)], 34, 1, 64, 32, 2),
    ([(200, 1), (2100, 300)], 56, 8, 128, 32, 3),
], ids=lambda v: "_".join("%d+%d" % x for x in v[:4]) if isinstance(v, list) else str(v))
def test_paged_chunks_and_mixed(seqs, H, KV, d, P, pad, alibi, dt):
    """Chunks short and long, alone and beside sequences that decode: the streaming kernel's one and two column tiles, the tile kernel, its splits, and both."""
    p = Paged(seqs, H, KV, d, P, dt, pad)
    check_attention(*p.run(alibi, max_q=max(q for _, q in seqs), max_kv=max(a + b for a, b in seqs)), what="chunks")


@pytest.mark.parametrize("hints", [(1, 1), (10000, 10**6), (None, None), (5, 100)], ids=str)
def test_paged_hints_do_not_change_the_result(hints):
    p = Paged([(300, 1), (0, 60), (1700, 2), (40, 17)], 8, 2, 128, 32, "fp16", 4)
    check_attention(*p.run(False, max_q=hints[0], max_kv=hints[1]), what="hints")


@pytest.mark.parametrize("n", [64, 257, 2048])
def test_paged_decode_many_sequences(n):
    r = random.Random(n)
    top = 500 if n < 1000 else 40
    check_attention(*Paged([(r.choice((0, 3, r.randint(0, top))), r.choice((1, 1, 1, 0))) for _ in range(n)], 4, 2, 64, 16, "bf16", 3).run(max_q=1), what="many")


@pytest.mark.parametrize("H,KV,d,dt,alibi", [(8, 1, 128, "fp16", False), (8, 2, 64, "bf16", True), (40, 2, 64, "fp16", False)])
def test_paged_parts_of_both_kernels(H, KV, d, dt, alibi):
    """Long contexts of few heads: single tokens' walks are cut among waves and a chunk's into key splits, each with its own part of the workspace; group 20: launched
    one after the other."""
    check_attention(*Paged([(9000, 1), (4000, 300), (0, 0), (7001, 2), (2500, 40)], H, KV, d, 16, dt, 5).run(alibi, max_q=300), what="parts of both")


def test_paged_mostly_idle_slots():
    """As many sequences as a call takes, nearly all of them without rows: far between two that have some, at the front and at the end; chunks among them."""
    for live, q in (((0, 1, 700, 2047), 1), ((64, 1500), 1), ((3, 900, 901, 2000), 50)):
        seqs = [(0, 0)] * 2048
        for i, s in enumerate(live):
            seqs[s] = (300 + 100 * i, q if i % 2 == 0 else 1)
        check_attention(*Paged(seqs, 4, 2, 64, 64, "fp16", 3).run(max_q=q, max_kv=800), what="idle")


def test_paged_long_context():
    """Many parts of one row tile, ids reloaded many times, small pages."""
    check_attention(*Paged([(40000, 1)], 4, 1, 128, 16, "fp16").run(max_q=1), what="long")
    check_attention(*Paged([(20011, 1), (5, 1), (9000, 1)], 6, 2, 64, 64, "bf16").run(True, max_q=1), what="long, ragged")
    check_attention(*Paged([(9000, 20)], 8, 1, 128, 16, "fp16").run(max_q=20), what="long chunk")


@pytest.mark.parametrize("q", [1, 3, 50])
def test_paged_rows_that_see_nothing(q):
    """No keys, fewer keys than new tokens, tables without pages: zeros, and the other sequences as ever."""
    p = Paged([(0, q), (20, q), (100, q), (0, q)], 4, 2, 64, 16, "fp16", 2)
    p.table[0] = [-1] * len(p.table[0])
    out, parts = p.run(max_q=q, kv_lens=[0, 20 + q, -3, max(q - 1, 0)])
    check_attention(out, parts, what="nothing to see")
    assert bool((out[:q] == 0).all()) and bool((out[2 * q:3 * q] == 0).all())


@pytest.mark.parametrize("alibi", [False, True], ids=["plain", "alibi"])
@pytest.mark.parametrize("q,P", [(1, 16), (1, 64), (3, 32), (60, 16), (150, 64)])
def test_paged_bad_pages_are_masked(q, P, alibi):
    """Ids that are no pages of the pool, at the front, in the middle and at the end, and lengths beyond the table."""
    p = Paged([(400, q), (333, q), (300, q)], 6, 2, 128, P, "fp16", 1, width_extra=0)
    p.table[0][0] = -1
    p.table[0][3] = p.n_pages
    p.table[1][2] = -2**31
    p.table[1][-2] = 2**31 - 1
    p.table[2] = [-5] * len(p.table[2])
    cap = len(p.table[0]) * P
    check_attention(*p.run(alibi, max_q=q), what="bad pages")
    check_attention(*p.run(alibi, max_q=q, kv_lens=[cap + 20, cap + 5, 10]), what="beyond the table")


@pytest.mark.parametrize("q,H,KV", [(1, 8, 2), (1, 4, 4), (4, 4, 2), (20, 4, 4), (100, 8, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_paged_stale_values_do_not_matter(q, H, KV, d):
    """NaN and infinities in every position that no sequence has: behind the last one in its page, and in pages of nobody."""
    import torch
    p = Paged([(37, q), (250, q), (1030, q), (0, q)], H, KV, d, 64, "fp16")
    want, _ = p.run(max_q=q)
    used = torch.zeros((p.n_pages, 64), dtype=torch.bool, device="cuda")
    for s, (past, n) in enumerate(p.seqs):
        for j in range(past + n):
            used[p.table[s][j // 64], j % 64] = True
    for pages, val in ((p.k, math.nan), (p.v, math.inf), (p.v, math.nan), (p.k, math.inf)):
        pages.copy_(torch.where(used[:, None, :, None], pages, torch.full_like(pages, val)))
        got, _ = p.run(max_q=q)
        assert torch.equal(got, want)


@pytest.mark.parametrize("q", [2, 4, 16, 40, 140])
@pytest.mark.parametrize("val", [math.nan, math.inf, -math.inf], ids=str)
def test_later_tokens_do_not_matter(q, val):
    """A value row of the newest token that is not finite: NaN or infinite for the tokens that see it, as without it for the others; the same for keys."""
    import torch
    past = 70
    for where in ("v", "k"):
        p = Paged([(past, q), (10, q)], 8, 2, 64, 16, "fp16")
        want, _ = p.run(max_q=q)
        j = past + q - 1
        getattr(p, where)[p.table[0][j // 16], :, j % 16] = val
        got, _ = p.run(max_q=q)
        assert torch.equal(got[q:], want[q:])
        assert torch.allclose(got[:q - 1].float(), want[:q - 1].float(), rtol=2.0**-9, atol=2.0**-10)
        if where == "v" or math.isnan(val):
            assert not bool(torch.isfinite(got[q - 1]).any())

    out, _ = packed_run([q, 30], 8, 1, 64, "bf16", False, edit=lambda x: x[q - 1, 9 * 64:].fill_(val))     # the first prompt's last value row
    ref, _ = packed_run([q, 30], 8, 1, 64, "bf16", False)
    assert torch.equal(out[q:], ref[q:])
    assert torch.allclose(out[:q - 1].float(), ref[:q - 1].float(), rtol=2.0**-6, atol=2.0**-7)
    assert not bool(torch.isfinite(out[q - 1]).any())


def odd_reference_of(plain):
    """attention_ref where values may be infinite or NaN: every weight is positive, so such a value makes its feature what it is itself, for the rows that see
    it and no others.  A weight that rounds to zero makes an infinity NaN in a product; beside a largest weight of 1 or more (E is then infinite) that is one of at
    most half of fp16's smallest step, 2^-25, or, in bf16, whose steps are smaller, one below 2^-126: the hardware's exponential has no subnormal results."""
    import torch

    def ref(q, k, v, ok, pos, slopes):
        fin, group, zero = torch.isfinite(v), q.shape[1] // k.shape[1], {torch.float16: 2.0**-25, torch.bfloat16: 2.0**-126}[q.dtype]
        out, A, E = plain(q, k, torch.where(fin, v, torch.zeros_like(v)), ok, pos, slopes)
        for j in torch.nonzero(~fin.all(2).all(1) & ok).flatten().tolist():
            sees = pos >= j
            rest = torch.where(fin[j], torch.zeros_like(v[j]), v[j]).double().repeat_interleave(group, 0)
            out[sees] += rest
            for t in torch.nonzero(sees).flatten().tolist():
                kt = k[:int(pos[t]) + 1].double().repeat_interleave(group, 1)
                s = (q[t].double()[None] * kt).sum(2) / math.sqrt(q.shape[2])
                if slopes is not None:
                    s = s + slopes.double()[None] * (torch.arange(len(kt), device="cuda") - pos[t]).double()[:, None]
                s[~ok[:len(kt)]] = -math.inf
                small = torch.exp(s[j] - s.amax(0)) <= 1.01 * zero
                E[t] = torch.where(small[:, None] & torch.isinf(rest), torch.full_like(E[t], math.inf), E[t])
        return out, A, E

    return ref


def check_odd(got, parts, what=""):
    import torch
    u = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}[got.dtype]
    for (r0, r1), (out, A, E) in parts:
        if r1 == r0:
            continue
        g, fin = got[r0:r1].double().view(out.shape), torch.isfinite(out)
        same = (g == out) | (torch.isnan(g) & (torch.isnan(out) | torch.isinf(E)))
        tol = u * (A + out.abs()) + E + u * (out.abs() + u * A + E) + 2.0**-25
        bad = torch.nonzero(~torch.where(fin, (g - out).abs() <= tol, same))
        assert bad.shape[0] == 0, "%s: rows %d..%d, %d elements, the first at %s" % (what, r0, r1, bad.shape[0], bad[0].tolist())


INF, NAN = math.inf, math.nan


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("past,q,H,KV,d,P,alibi", [
    (200, 1, 8, 2, 64, 16, False), (70, 3, 8, 2, 128, 16, True), (0, 4, 4, 4, 64, 64, False), (900, 16, 4, 2, 128, 32, False), (31, 12, 34, 17, 64, 16, True),
    (40, 33, 2, 2, 128, 16, False), (100, 140, 8, 2, 64, 64, True), (2000, 60, 4, 1, 128, 32, False), (0, 300, 3, 3, 128, 16, True), (250, 270, 2, 1, 64, 256, False),
])
def test_infinite_values_reach_the_rows_that_see_them(past, q, H, KV, d, P, alibi, dt, monkeypatch):
    """Single infinite and NaN elements of values: in the first position, in cached ones, in the new tokens' own from the first to the last."""
    import torch
    p = Paged([(past, q), (past // 2, q), (5, 1)], H, KV, d, P, dt, 2)
    p.qkv[:, :H * d] *= 0.125
    r = random.Random(past + q)
    new = sorted({past, past + q // 2, past + q // 3, past + q - 1, past + r.randrange(q)})
    for n, j in enumerate([0, past // 3] + new):
        for val in (INF, -INF, NAN)[n % 3:][:2]:
            p.v[p.table[0][j // P], r.randrange(KV), j % P, r.randrange(d)] = val
    monkeypatch.setitem(globals(), "attention_ref", odd_reference_of(attention_ref))
    check_odd(*p.run(alibi, max_q=q), what="paged")


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,H,KV,d,alibi", [([5, 40], 4, 2, 64, False), ([130, 64, 1], 4, 4, 128, True), ([300, 17], 6, 2, 128, False), ([513], 20, 4, 64, True), ([90, 200], 40, 1, 64, False)])
def test_infinite_values_of_packed_rows(lens, H, KV, d, alibi, dt, monkeypatch):
    import torch
    r = random.Random(sum(lens))

    def edit(x):
        x[:, :H * d] *= 0.125
        cu = np.concatenate([[0], np.cumsum(lens)])
        for s, n in enumerate(lens):
            for i, j in enumerate(sorted({0, n // 2, n - 1, r.randrange(n), r.randrange(n)})):
                x[cu[s] + j, (H + KV) * d + r.randrange(KV * d)] = (INF, -INF, NAN)[i % 3]

    monkeypatch.setitem(globals(), "attention_ref", odd_reference_of(attention_ref))
    check_odd(*packed_run(lens, H, KV, d, dt, alibi, 1, edit=edit), what="packed %s" % lens)


def test_an_infinite_value_costs_little():
    """One infinite element in the first value row, which every row sees; and one in every value row, so that some are at every diagonal."""
    import torch
    H, KV, d, n = 8, 2, 128, 3000

    def time_of(call):
        for _ in range(2):
            call()
        torch.cuda.synchronize()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(3):
            call()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / 3

    qkv = torch.randn((n, (H + 2 * KV) * d), generator=gen(1), device="cuda").half()
    k, v = (torch.randn((n // 16 + 1, KV, 16, d), generator=gen(2 + i), device="cuda").half() for i in range(2))
    table, cu = ints([list(range(n // 16 + 1))]), ints([0, n])
    few, cu_few, kv = qkv[:4].contiguous(), ints([0, 4]), ints([n])
    calls = (lambda: lpq.lpq_packed_attention(qkv, cu, H, KV), lambda: lpq.lpq_paged_attention(qkv, k, v, table, cu, kv),
             lambda: lpq.lpq_paged_attention(few, k, v, table, cu_few, kv))
    plain = [time_of(c) for c in calls]
    qkv[0, (H + KV) * d + 3] = v[0, :, 0, 3] = INF
    first = [time_of(c) for c in calls]
    qkv[:, (H + KV) * d + 3] = v[:, :, :, 3] = INF
    every = [time_of(c) for c in calls]
    print("ms without, one, in every row:", plain, first, every)
    assert all(b <= 5 * a for a, b in zip(plain, first)), (plain, first)
    assert all(b <= 50 * a for a, b in zip(plain, every)), (plain, every)


def test_nan_throughout():
    """A batch whose values, or queries, are NaN everywhere: NaN everywhere, and no row is walked to its end on the way."""
    import torch
    for where in ("v", "qkv"):
        p = Paged([(2000, 900), (700, 3), (50, 1)], 8, 2, 128, 64, "bf16")
        getattr(p, where).fill_(math.nan)
        out = torch.zeros((p.M, 8 * 128), dtype=torch.bfloat16, device="cuda")
        lpq.lpq_paged_attention(p.qkv, p.k, p.v, ints(p.table), ints(p.cu), ints([a + b for a, b in p.seqs]), max_q=900, out=out)
        assert bool(torch.isnan(out).all())
    out = lpq.lpq_packed_attention(torch.full((2500, 12 * 64), math.nan, dtype=torch.float16, device="cuda"), ints([0, 2400, 2500]), 8, 2)
    assert bool(torch.isnan(out).all())


def test_large_scores():
    """Scores in the thousands: one key takes all; and all scores equal."""
    import torch
    p = Paged([(500, 1), (300, 30)], 4, 2, 128, 32, "fp16")
    p.qkv *= 20
    check_attention(*p.run(max_q=30), what="large")
    p.k.zero_()
    check_attention(*p.run(max_q=30), what="equal")


@pytest.mark.parametrize("biases", [False, True], ids=["plain", "biases"])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_beyond_24_bits(d, dt, biases):
    """Scores so large that neighbours in 32 bits are tens or hundreds apart, each of them exact: the visible keys with the largest share the weight equally, the
    others have none.  Off by the output's rounding, and 2^-20 for 32-bit sums and the division; the weights are equal, so their rounding is gone.  (With biases
    of zero: the kernels' other form.)"""
    import torch
    u, r = {"fp16": 2.0**-11, "bf16": 2.0**-8}[dt], random.Random(d)
    seqs, H, KV = [(300, 1), (0, 300), (70, 90), (500, 6), (0, 1), (64, 17)], 4, 2
    for max_q, step in ((300, 2048.0), (300, 4.0), (6, 2048.0)):
        p = Paged([(a, min(b, max_q)) for a, b in seqs], H, KV, d, 32, dt, 1)
        p.qkv[:, :H * d] = 16384.0
        levels = [torch.tensor([r.randint(-7, 7) for _ in range(a + b)], device="cuda") for a, b in p.seqs]
        for s, lv in enumerate(levels):
            for i in range(0, len(lv), 32):
                n = min(32, len(lv) - i)
                p.k[p.table[s][i // 32], :, :n] = (lv[i:i + n] * step).to(p.k.dtype)[None, :, None]
        out = torch.full((p.M, H * d), 77.0, dtype=p.qkv.dtype, device="cuda")
        slopes = torch.zeros(H, device="cuda") if biases else None
        lpq.lpq_paged_attention(p.qkv, p.k, p.v, ints(p.table), ints(p.cu), ints([a + b for a, b in p.seqs]), max_q=max_q, alibi_slopes=slopes, out=out)
        for s, (past, n) in enumerate(p.seqs):
            L = past + n
            v = p.v[torch.tensor([p.table[s][j // 32] for j in range(L)], device="cuda"), :, torch.arange(L, device="cuda") % 32].double()
            for t in range(n):
                seen = levels[s][:past + t + 1]
                rows = v[:past + t + 1][seen == seen.max()].repeat_interleave(H // KV, 1)
                want, size = rows.mean(0), rows.abs().mean(0)
                err = (out[p.cu[s] + t].double().view(H, d) - want).abs()
                assert bool((err <= u * want.abs() + 2.0**-20 * size + 2.0**-25).all()), (max_q, step, s, t, float(err.max()))


@pytest.mark.parametrize("biases", [False, True], ids=["plain", "biases"])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_many_small_weights(dt, biases):
    """One key that outweighs each of the others by 2^25.5, which is less than fp16's smallest step beside it, with a value of zero, and thousands of others, with
    ones.  Off by the weights' and the output's rounding (2 u of the result), exponents of 25.5 from exact 32-bit products (2^-12) and 32-bit sums (2 n 2^-24)."""
    import torch
    u, H, KV, d = {"fp16": 2.0**-11, "bf16": 2.0**-8}[dt], 4, 2, 64
    for past, n in ((60000, 1), (30000, 3), (9000, 64), (3000, 300)):
        p = Paged([(past, n)], H, KV, d, 64, dt)
        p.qkv.zero_(), p.k.zero_(), p.v.fill_(1.0)
        p.qkv[:, :H * d:d] = 16.0
        at = past // 3
        p.k[p.table[0][at // 64], :, at % 64, 0] = 8.84375                      # a score of 17.6875, in bf16 of 17.75
        p.v[p.table[0][at // 64], :, at % 64] = 0.0
        out = torch.full((p.M, H * d), 77.0, dtype=p.qkv.dtype, device="cuda")
        lpq.lpq_paged_attention(p.qkv, p.k, p.v, ints(p.table), ints(p.cu), ints([past + n]), max_q=n, alibi_slopes=torch.zeros(H, device="cuda") if biases else None, out=out)
        rest = (past + torch.arange(n, device="cuda").double()) * math.exp(-2 * float(p.k[p.table[0][at // 64], 0, at % 64, 0]))
        want = (rest / (1 + rest))[:, None]
        assert bool(((out.double() - want).abs() <= (2 * u + 2.0**-12 + 2 * (past + n) * 2.0**-24) * want + 2.0**-25).all()), (past, n, float(out.min()), float(want.min()))


def test_pool_past_32_bits():
    """Pages more than 2^31 elements into the pool."""
    import torch
    P, KV, d = 256, 16, 128
    n_pages = 2**31 // (KV * P * d) + 40
    k, v = (torch.zeros((n_pages, KV, P, d), dtype=torch.float16, device="cuda") for _ in range(2))
    p = Paged([(700, 1), (100, 40)], 16, KV, d, P, "fp16")
    off = n_pages - p.n_pages
    k[off:], v[off:] = p.k, p.v
    want, parts = p.run(max_q=40)
    p.table = [[t + off if t >= 0 else t for t in row] for row in p.table]
    p.k, p.v, p.n_pages = k, v, n_pages
    got, _ = p.run(max_q=40)
    assert torch.equal(got, want)
    slots = [(n_pages - 1) * P + 255, 3]
    rows = p.qkv[:2].contiguous()
    lpq.lpq_paged_append(rows, k, v, ints(slots))
    assert torch.equal(k[n_pages - 1, :, 255], rows[0, 16 * d:32 * d].view(KV, d)) and torch.equal(v[0, :, 3], rows[1, 32 * d:].view(KV, d))


def test_same_inputs_same_bits():
    import torch
    p = Paged([(3000, 1), (700, 60), (10, 1)], 8, 2, 128, 16, "fp16")
    a, _ = p.run(max_q=60)
    for _ in range(3):
        assert torch.equal(p.run(max_q=60)[0], a)


def test_binding_checks():
    import torch
    p = Paged([(30, 1), (20, 1)], 4, 2, 64, 16, "fp16")
    t, cu, kv = ints(p.table), ints(p.cu), ints([31, 21])
    call = lambda **k: lpq.lpq_paged_attention(**{**dict(qkv=p.qkv, k_pages=p.k, v_pages=p.v, table=t, cu_q=cu, kv_lens=kv), **k})
    call()
    for bad in (dict(qkv=p.qkv.bfloat16()), dict(qkv=p.qkv[:, :-8].contiguous()), dict(k_pages=p.k[:, :1].contiguous()), dict(v_pages=p.v[1:]), dict(table=t.long()),
                dict(table=t[:1]), dict(cu_q=cu[:2]), dict(kv_lens=kv.cpu()), dict(table=t.t()), dict(out=p.qkv), dict(out=torch.zeros((2, 256), device="cuda")),
                dict(alibi_slopes=torch.ones(3, device="cuda")), dict(qkv=p.qkv.cpu())):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(max_q=0), dict(max_kv=0), dict(qkv=p.qkv[:, :-64].contiguous())):      # 3 heads over 2 K/V heads
        with pytest.raises(lpq.LpqError):
            call(**bad)
    with pytest.raises(ValueError):
        lpq.lpq_paged_append(p.qkv, p.k, p.v, ints([1]))
    with pytest.raises(ValueError):
        lpq.lpq_paged_plan(kv, kv, t, ints([0] * 9), ints([0, 9, 1]), 16, 2)
    with pytest.raises(ValueError):
        lpq.lpq_packed_attention(p.qkv, cu, 3, 2)


# ---- a run of them together -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("alibi", [False, True], ids=["plain", "alibi"])
def test_serving_run(alibi):
    """Requests come, are prefilled (whole and in chunks) and decode side by side through a quantised QKV linear; some finish, their pages go to others.
    Every step's output against 64 bits on the step's own qkv and all the keys and values appended so far."""
    import torch
    H, KV, d, P, n_pages, width, N, M = 8, 2, 64, 16, 40, 12, 6, 96
    cols = (H + 2 * KV) * d
    g = gen(5)
    w = lpq.lpq_quantize_pack((torch.randn((cols, H * d), generator=g, device="cuda") * 0.06).half(), 4, lpq.LPQ_ASYM_GROUP)
    k, v = (torch.full((n_pages, KV, P, d), math.nan, dtype=torch.float16, device="cuda") for _ in range(2))
    table, ring, counters = torch.full((N, width), -1, dtype=torch.int32, device="cuda"), torch.arange(n_pages, dtype=torch.int32, device="cuda"), ints([0, n_pages])
    lens = torch.zeros(N, dtype=torch.int32, device="cuda")
    plan = None
    history = [([], []) for _ in range(N)]
    steps = [[50, 0, 20, 0, 0, 0], [1, 30, 1, 40, 0, 0], [1, 1, 1, 30, 9, 0], [1, 1, -1, 1, 1, 60], [1, -1, 25, 1, 1, 20], [1, 33, 1, -1, 30, 1], [40, 1, 1, 45, 1, 1], [1, 1, 1, 1, 1, 1]]
    slopes = slopes_of(H, alibi)
    for step, q in enumerate(steps):
        x = torch.randn((M, H * d), generator=g, device="cuda").half()
        qkv = lpq.lpq_qlinear_fused(w, x, lpq.LPQ_PREFILL)
        plan = lpq.lpq_paged_plan(lens, ints(q), table, ring, counters, P, M, plan=None if plan is None else plan)
        if plan.kv_lens.data_ptr() != lens.data_ptr():
            lens.copy_(plan.kv_lens), counters.copy_(plan.counters)
            plan = plan._replace(kv_lens=lens, counters=counters)          # in place from now on
        lpq.lpq_paged_append(qkv, k, v, plan.slots)
        out = torch.full((M, H * d), 77.0, dtype=torch.float16, device="cuda")
        lpq.lpq_paged_attention(qkv, k, v, table, plan.cu_q, lens, max_q=max(q), alibi_slopes=slopes, out=out)
        assert plan.info[3].item() == 0, "the pool is large enough for these requests"
        parts, r0 = [], 0
        for s, n in enumerate(q):
            if n < 0:
                history[s] = ([], [])
                continue
            rows = qkv[r0:r0 + n]
            history[s][0].append(rows[:, H * d:(H + KV) * d].reshape(n, KV, d)), history[s][1].append(rows[:, (H + KV) * d:].reshape(n, KV, d))
            ks, vs = torch.cat(history[s][0]), torch.cat(history[s][1])
            L = ks.shape[0]
            assert lens[s].item() == L
            parts.append(((r0, r0 + n), attention_ref(rows[:, :H * d].reshape(n, H, d), ks, vs, torch.ones(L, dtype=torch.bool, device="cuda"),
                                                      L - n + torch.arange(n, device="cuda"), slopes)))
            r0 += n
        check_attention(out, parts, what="step %d" % step)
    held = sum(-(-int(n) // P) for n in lens.tolist())
    assert counters[1].item() == n_pages - held
    # every page is somebody's or free, none twice
    head, free = counters.tolist()
    owned = [t for s in range(N) for t in table[s, :-(-int(lens[s]) // P)].tolist()]
    assert sorted(owned + [ring[(head + i) % n_pages].item() for i in range(free)]) == list(range(n_pages))


@pytest.mark.parametrize("q", [1, 5, 40])
def test_starved_sequences_beside_served_ones(q):
    """A step with too few pages: served sequences are exact, nothing of a starved one is written anywhere but in its own output rows, which are its queries' over
    the cached positions; with pages returned the same step is exact for it too."""
    import torch
    H, KV, d, P, n_pages = 8, 2, 64, 16, 30
    past, lens = [80, 64, 0, 70], [0, q, q, q]                      # the second and third need pages, the fourth (one token) may not
    held = [-(-p // P) for p in past]
    need = [-(-(p + n) // P) - h for p, n, h in zip(past, lens, held)]
    g = gen(q)
    k, v = (torch.randn((n_pages, KV, P, d), generator=g, device="cuda").half() for _ in range(2))
    ids = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-1] * (10 - h))
        at += h
    free = need[1]                                                  # the second's
    ring = ids[at:] + [-1] * at
    table_d, ring_d, counters, M = ints(table), ints(ring), ints([0, free]), 3 * q + 2
    qkv = torch.randn((M, (H + 2 * KV) * d), generator=g, device="cuda").half()
    k0, v0 = k.clone(), v.clone()
    plan = lpq.lpq_paged_plan(ints(past), ints(lens), table_d, ring_d, counters, P, M)
    starved = [s for s in range(4) if lens[s] and need[s] and s > 1]
    assert 2 in starved and plan.info.tolist()[3] == len(starved)
    cu, kv, slots = plan.cu_q.tolist(), plan.kv_lens.tolist(), plan.slots.tolist()
    for s in range(4):
        assert (kv[s] == past[s]) == (s in starved or not lens[s]) and all((x == -1) == (s in starved) for x in slots[cu[s]:cu[s + 1]])
    lpq.lpq_paged_append(qkv, k, v, plan.slots)
    mine = torch.zeros((n_pages, P), dtype=torch.bool, device="cuda")
    for x in slots:
        if x >= 0:
            mine[x // P, x % P] = True
    assert torch.equal(torch.where(mine[:, None, :, None], k0, k), k0) and torch.equal(torch.where(mine[:, None, :, None], v0, v), v0)

    def check(out, kv, cu):
        rows = table_d.tolist()
        parts = []
        for s in range(4):
            L, r0, r1 = kv[s], cu[s], cu[s + 1]
            page = torch.tensor([rows[s][j // P] for j in range(L)], dtype=torch.long, device="cuda")
            off = torch.arange(L, device="cuda") % P
            parts.append(((r0, r1), attention_ref(qkv[r0:r1, :H * d].view(r1 - r0, H, d), k[page, :, off], v[page, :, off], page >= 0, L - (r1 - r0) + torch.arange(r1 - r0, device="cuda"), None)))
        check_attention(out, parts, what="starved")

    out = torch.full((M, H * d), 77.0, dtype=torch.float16, device="cuda")
    lpq.lpq_paged_attention(qkv, k, v, table_d, plan.cu_q, plan.kv_lens, max_q=q, out=out)
    check(out, kv, cu)
    assert bool((out[cu[2]:cu[3]] == 0).all())                      # nothing cached
    # the first sequence has finished: its pages serve the starved in the step after
    back = lpq.lpq_paged_plan(plan.kv_lens, ints([-1, 0, 0, 0]), table_d, ring_d, plan.counters, P, M)
    assert back.info.tolist() == [0, 0, held[0], 0]
    again = [0, 0] + [lens[s] if s in starved else 0 for s in (2, 3)]
    plan = lpq.lpq_paged_plan(back.kv_lens, ints(again), table_d, ring_d, back.counters, P, M)
    assert plan.info.tolist()[3] == 0
    cu, kv = plan.cu_q.tolist(), plan.kv_lens.tolist()
    lpq.lpq_paged_append(qkv, k, v, plan.slots)
    out = torch.full((M, H * d), 77.0, dtype=torch.float16, device="cuda")
    lpq.lpq_paged_attention(qkv, k, v, table_d, plan.cu_q, plan.kv_lens, max_q=q, out=out)
    check(out, kv, cu)


def test_paged_against_packed_and_contiguous():
    """The same prompts through the packed rows, through pages, and (one length, as many K/V heads as heads) through the contiguous cache."""
    import torch
    H, d, T, B, P = 5, 128, 150, 3, 32
    qkv = torch.randn((B * T, 3 * H * d), generator=gen(9), device="cuda").half()
    one = torch.ones(H * d, dtype=torch.float16, device="cuda")
    st = lpq.LayerState(H, d, 192, B, torch.device("cuda"), (one, one), (one, one))
    lpq.lpq_kv_append(qkv, st, B, T, 0)
    want = lpq.lpq_attention(qkv, st, B, T, 0).float()
    cu = ints([0, T, 2 * T, 3 * T])
    table, ring = torch.full((B, 5), -1, dtype=torch.int32, device="cuda"), torch.arange(20, dtype=torch.int32, device="cuda").flip(0).contiguous()
    plan = lpq.lpq_paged_plan(ints([0] * B), ints([T] * B), table, ring, ints([0, 20]), P, B * T)
    assert torch.equal(plan.cu_q, cu)
    k, v = (torch.zeros((20, H, P, d), dtype=torch.float16, device="cuda") for _ in range(2))
    lpq.lpq_paged_append(qkv, k, v, plan.slots)
    # each side is within its rounding of the exact result: weights and output in fp16, |v| up to about 4.5
    for got in (lpq.lpq_packed_attention(qkv, cu, H, H), lpq.lpq_paged_attention(qkv, k, v, table, cu, plan.kv_lens)):
        assert float((got.float() - want).abs().max()) <= 2 * 2 * 2.0**-11 * 4.5


# ---- streams and graphs -----------------------------------------------------------------------------------------------

def test_on_another_stream():
    import torch
    p = Paged([(900, 1), (40, 30)], 8, 2, 64, 16, "fp16")
    want, _ = p.run(max_q=30)
    s = torch.cuda.Stream()
    t, cu, kv, out = ints(p.table), ints(p.cu), ints([901, 70]), torch.full_like(want, 77.0)
    torch.cuda.synchronize()
    lpq.lpq_paged_attention(p.qkv, p.k, p.v, t, cu, kv, max_q=30, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


def test_on_another_stream_with_new_outputs():
    """Outputs that the binding makes, on a stream of the caller's while the current one is busy: what is filled or still in use on the current one must not
    reach them, neither while it works nor afterwards."""
    import torch
    p = Paged([(900, 1), (40, 30)], 8, 2, 64, 16, "fp16", 3)
    want, _ = p.run(max_q=30)
    want[31:] = 0
    t, cu, kv = ints(p.table), ints(p.cu), ints([901, 70])
    packed = lpq.lpq_packed_attention(p.qkv, ints([0, 34]), 8, 2)
    case = plan_case(3, 40, 32, MIXED, 300, 5)
    past, q, table, ring, counters, M = ints(case[0]), ints(case[1]), ints(case[2]), ints(case[3]), ints(case[4:6]), case[6]
    plan = lpq.lpq_paged_plan(past, q, table.clone(), ring.clone(), counters, 32, M)
    s, cu2 = torch.cuda.Stream(), ints([0, 34])
    torch.cuda.synchronize()
    calls = [(lambda: [lpq.lpq_paged_attention(p.qkv, p.k, p.v, t, cu, kv, max_q=30, stream=s)], [want]),
             (lambda: [lpq.lpq_packed_attention(p.qkv, cu2, 8, 2, stream=s)], [packed]),
             (lambda: list(lpq.lpq_paged_plan(past, q, table, ring, counters, 32, M, stream=s)), list(plan))]
    for call, expected in calls:
        freed = [torch.empty_like(e) for e in expected]
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        for f in freed:
            f.fill_(-9)                                # queued behind the sleep, in memory that is free for the current stream's next tensors
        del freed, f
        got = call()
        s.synchronize()
        with torch.cuda.stream(s):
            assert all(torch.equal(g, e) for g, e in zip(got, expected))
        torch.cuda.synchronize()
        assert all(torch.equal(g, e) for g, e in zip(got, expected))


def test_long_plan_beside_attention():
    """Plans of more rows than one launch takes on a stream of their own, while attention with partial results runs on another: both as by themselves."""
    import torch
    p = Paged([(5000, 1), (2000, 40), (700, 1)], 8, 2, 128, 16, "fp16")
    want, _ = p.run(max_q=40)
    t, cu, kv, out = ints(p.table), ints(p.cu), ints([5001, 2040, 701]), torch.full_like(want, 77.0)
    case = plan_case(6, 40, 32, lambda r: r.randint(300, 600), 400, 9)
    ref = plan_ref(*case[:6], 32, case[6])
    past, q, M = ints(case[0]), ints(case[1]), case[6]
    assert M > 10000
    inputs = [(ints(case[2]), ints(case[3]), ints(case[4:6])) for _ in range(20)]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    plans = []
    for table, ring, counters in inputs:
        lpq.lpq_paged_attention(p.qkv, p.k, p.v, t, cu, kv, max_q=40, out=out, stream=a)
        plans.append(lpq.lpq_paged_plan(past, q, table, ring, counters, 32, M, stream=b))
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    for plan, (table, ring, _) in zip(plans, inputs):
        got = dict({k: getattr(plan, k).tolist() for k in plan._fields}, table=table.tolist(), ring=ring.tolist())
        for name in ref:
            assert got[name] == ref[name], name


def test_captured_decode_loop():
    """A decode step (plan in place, append, attention) captured once and replayed: each replay is the next step, as the eager loop has it; eager work of other
    sizes, with its own use of the workspace, runs between the replays."""
    import torch
    H, KV, d, P, N, n_pages = 8, 2, 128, 16, 5, 80

    def fresh():
        g = gen(3)
        return dict(k=torch.zeros((n_pages, KV, P, d), dtype=torch.float16, device="cuda"), v=torch.zeros((n_pages, KV, P, d), dtype=torch.float16, device="cuda"),
                    table=torch.full((N, 14), -1, dtype=torch.int32, device="cuda"), ring=torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32),
                    counters=ints([7, n_pages]), lens=ints([0] * N), q=ints([60, 15, 16, 131, 1]), x=torch.zeros((230, (H + 2 * KV) * d), dtype=torch.float16, device="cuda"),
                    out=torch.zeros((230, H * d), dtype=torch.float16, device="cuda"),
                    plan=[torch.empty(m, dtype=torch.int32, device="cuda") for m in (N + 1, N, 230, 230, 2, 4)])

    def step(s, max_q):
        plan = (s["plan"][0], s["lens"], s["plan"][2], s["plan"][3], s["counters"], s["plan"][5])
        lpq.lpq_paged_plan(s["lens"], s["q"], s["table"], s["ring"], s["counters"], P, 230, plan=plan)
        lpq.lpq_paged_append(s["x"], s["k"], s["v"], s["plan"][2])
        lpq.lpq_paged_attention(s["x"], s["k"], s["v"], s["table"], s["plan"][0], s["lens"], max_q=max_q, max_kv=14 * P, out=s["out"])

    xs = [torch.randn((230, (H + 2 * KV) * d), generator=gen(50 + i), device="cuda").half() for i in range(6)]
    eager, want = fresh(), []
    for i, x in enumerate(xs):
        eager["x"].copy_(x)
        step(eager, 131 if i == 0 else 1)
        want.append(eager["out"].clone())
        eager["q"].fill_(1)
    s = fresh()
    s["x"].copy_(xs[0])
    step(s, 131)
    assert torch.equal(s["out"], want[0])
    s["q"].fill_(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s, 1)
    other = Paged([(3000, 1), (100, 40)], 8, 2, 128, 32, "fp16")
    other_want, _ = other.run(max_q=40)
    for i in range(1, 6):
        s["x"].copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s["out"], want[i]), "replay %d" % i
        assert torch.equal(other.run(max_q=40)[0], other_want)
    for name in ("k", "v", "table", "ring", "counters", "lens"):
        assert torch.equal(s[name], eager[name]), name


def test_captured_steps_of_all_kinds():
    """Plan of more rows than one launch takes, append, mixed paged and packed attention, captured once: replays with other lengths (sequences that decode become
    chunks and the other way round), eager calls with workspace between them, against the same calls made eagerly."""
    import torch
    H, KV, d, P, N, M, n_pages = 8, 2, 128, 16, 4, 7000, 400
    x = torch.randn((M, (H + 2 * KV) * d), generator=gen(1), device="cuda").half()
    base_k, base_v = (torch.randn((n_pages, KV, P, d), generator=gen(2 + i), device="cuda").half() for i in range(2))
    ring = torch.randperm(n_pages, generator=gen(4), device="cuda").to(torch.int32)
    slopes = slopes_of(H, True)

    def fresh():
        return dict(k=base_k.clone(), v=base_v.clone(), table=torch.full((N, 140), -1, dtype=torch.int32, device="cuda"), ring=ring.clone(), counters=ints([0, n_pages]),
                    lens=ints([0] * N), q=ints([0] * N), plan=[torch.zeros(m, dtype=torch.int32, device="cuda") for m in (N + 1, N, M, M, 2, 4)],
                    out=torch.zeros((M, H * d), dtype=torch.float16, device="cuda"), packed=torch.zeros((M, H * d), dtype=torch.float16, device="cuda"))

    def step(s):
        plan = (s["plan"][0], s["lens"], s["plan"][2], s["plan"][3], s["counters"], s["plan"][5])
        lpq.lpq_paged_plan(s["lens"], s["q"], s["table"], s["ring"], s["counters"], P, M, plan=plan)
        lpq.lpq_paged_append(x, s["k"], s["v"], s["plan"][2])
        lpq.lpq_paged_attention(x, s["k"], s["v"], s["table"], s["plan"][0], s["lens"], max_q=1500, max_kv=2000, alibi_slopes=slopes, out=s["out"])
        lpq.lpq_packed_attention(x, s["plan"][0], H, KV, max_q=1500, out=s["packed"])

    steps = [[1500, 20, 0, 300], [1, 1, 900, 1], [1, 200, 40, 1], [-1, 1, 1, 500], [600, 1, -1, 1], [1, 1, 5, 1]]
    eager, want = fresh(), []
    for q in steps:
        eager["q"].copy_(ints(q))
        step(eager)
        want.append([eager[n].clone() for n in ("out", "packed", "lens", "counters", "table", "ring")] + [t.clone() for t in (eager["plan"][0], eager["plan"][2], eager["plan"][3], eager["plan"][5])])
    assert all(w[-1][3].item() == 0 for w in want)
    s = fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s)
    other = Paged([(3000, 1), (100, 40)], 8, 2, 128, 32, "fp16")
    other_want, _ = other.run(max_q=40)
    for q, w in zip(steps, want):
        s["q"].copy_(ints(q))
        graph.replay()
        torch.cuda.synchronize()
        got = [s[n] for n in ("out", "packed", "lens", "counters", "table", "ring")] + [s["plan"][i] for i in (0, 2, 3, 5)]
        assert all(torch.equal(a, b) for a, b in zip(got, w)), q
        assert torch.equal(other.run(max_q=40)[0], other_want)
