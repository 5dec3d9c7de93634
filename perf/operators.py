"""Operators for batches of sequences of different lengths over a paged cache, as measurable cases.

A program that serves requests as they come keeps the K and V of all of them in a pool of pages.  Each step it plans where the
step's new tokens go (block tables and slots, on the GPU, from the lengths alone), appends their K and V to the pages, and lets the
new tokens attend: to their sequence's pages, be they one token each, chunks of prompts, or both in one batch; or, for whole
prompts, to the packed rows themselves.  The kinds below are those calls:

    plan      lpq_paged_plan       block tables, slots, positions and offsets of a step's rows from the requests' lengths
    append    lpq_paged_append     K and V of the rows into their slots
    packed    lpq_packed_attention causal attention of whole prompts, packed one behind the other
    paged     lpq_paged_attention  causal attention of new tokens over the pages of their sequences

Head layouts are the ones this repository's configurations have (hidden sizes 768, 5120, 7168, 9216 in heads of 64 or 128) and the same
with fewer heads of keys and values.  Lengths are a fixed function of a case's numbers; values are drawn from the seed: q, k and v
N(0, 1), q twice that, stale values in the pages' unused positions.
"""
import math
import random

import torch

own = False
DEVICE = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # a handful of users, one token each: the smallest step there is
        dict(name="plan_7seq_decode", kind="plan", decode=7, chunks=0, chunk=0, done=0, lo=20, hi=600, page=64, pad=1, shape=1),
        # a busy server's step: decoding, some prompts in chunks, some requests just finished; small pages
        dict(name="plan_300seq_mixed", kind="plan", decode=280, chunks=9, chunk=512, done=11, lo=16, hi=4000, page=16, pad=77, shape=2),
        # many long prompts admitted at once
        dict(name="plan_24prompts", kind="plan", decode=0, chunks=24, chunk=1100, done=0, lo=0, hi=0, page=32, pad=0, shape=3),
        # a decode step's append, every head with its own keys and values (7168 wide)
        dict(name="append_43row_56kv", kind="append", heads=56, kv=56, d=128, dtype="fp16", decode=43, chunks=0, chunk=0, lo=30, hi=300, page=64, pad=5, shape=4),
        # the append of a prefill step of several prompts, few heads of keys and values
        dict(name="append_prompts_8kv", kind="append", heads=64, kv=8, d=128, dtype="bf16", decode=0, chunks=5, chunk=1601, lo=0, hi=0, page=128, pad=0, shape=5),
        # the smallest model's prompts, shorter than a tile most of them
        dict(name="packed_768_9short", kind="packed", heads=12, kv=12, d=64, dtype="fp16", prompts=9, lo=1, hi=140, alibi=False, pad=11, shape=6),
        # a prefill micro-batch of the benchmark's width, ragged, with linear biases
        dict(name="packed_5120_4ragged", kind="packed", heads=40, kv=40, d=128, dtype="fp16", prompts=4, lo=300, hi=1500, alibi=True, pad=0, shape=7),
        # one long prompt, eight query heads to each head of keys and values
        dict(name="packed_8192_long_gqa8", kind="packed", heads=64, kv=8, d=128, dtype="bf16", prompts=1, lo=5801, hi=5801, alibi=False, pad=0, shape=8),
        # the benchmark's decode step: 16 sequences half way through their answers
        dict(name="paged_5120_16seq_decode", kind="paged", heads=40, kv=40, d=128, dtype="fp16", decode=16, chunks=0, chunk=0, lo=400, hi=700, page=64, alibi=False, pad=0, shape=9),
        # a busy server's decode step: contexts of all lengths, small pages, grouped heads
        dict(name="paged_8192_61seq_gqa8", kind="paged", heads=64, kv=8, d=128, dtype="bf16", decode=61, chunks=0, chunk=0, lo=100, hi=7000, page=16, alibi=False, pad=3, shape=10),
        # one user with a whole book as context
        dict(name="paged_7168_1seq_long", kind="paged", heads=56, kv=8, d=128, dtype="fp16", decode=1, chunks=0, chunk=0, lo=90001, hi=90001, page=128, alibi=False, pad=0, shape=11),
        # a mixed step: chunks of two long prompts beside sequences that decode
        dict(name="paged_7168_mixed_chunks", kind="paged", heads=56, kv=8, d=128, dtype="fp16", decode=9, chunks=2, chunk=512, lo=900, hi=6000, page=32, alibi=True, pad=13, shape=12),
    ]


HEADS = ((12, 12, 64), (12, 4, 64), (16, 2, 64), (40, 40, 128), (40, 8, 128), (56, 56, 128), (56, 8, 128), (64, 8, 128), (72, 8, 128))
PAGES = (16, 32, 64, 128, 256)


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("plan", "append", "packed", "packed", "paged", "paged", "paged"))
    shape = rng.randrange(1000, 1 << 30)
    if kind == "plan":
        decode, chunks, done = (rng.choice((0, _logu(rng, 1, top))) for top in (1000, 24, 40))
        return dict(kind=kind, decode=decode + 1, chunks=chunks, chunk=_logu(rng, 2, 1200), done=done, lo=rng.choice((0, 1, 50)), hi=_logu(rng, 60, 8000),
                    page=rng.choice(PAGES), pad=rng.choice((0, _logu(rng, 1, 300))), shape=shape)
    heads, kv, d = rng.choice(HEADS)
    case = dict(kind=kind, heads=heads, kv=kv, d=d, dtype=rng.choice(("fp16", "bf16")), pad=rng.choice((0, _logu(rng, 1, 40))), shape=shape)
    if kind == "packed":
        prompts = _logu(rng, 1, 16)
        hi = _logu(rng, 8, min(5800, math.sqrt(2.0e9 / (prompts * heads))))      # padded scores of the plain form: at most 8 GB
        return dict(case, prompts=prompts, lo=rng.randrange(1, hi + 1), hi=hi, alibi=rng.random() < 0.4)
    case["page"] = rng.choice(PAGES)
    if kind == "append":
        decode, chunks = rng.choice(((_logu(rng, 1, 200), 0), (0, _logu(rng, 1, 6)), (_logu(rng, 1, 60), _logu(rng, 1, 3))))
        return dict(case, decode=decode, chunks=chunks, chunk=_logu(rng, 2, 1600), lo=rng.choice((0, 33)),
                    hi=_logu(rng, 40, max(41, min(1500, 15e6 / (decode + chunks) / (kv * d)))))
    form = rng.choice(("decode", "decode", "chunks", "mixed"))
    decode = 0 if form == "chunks" else _logu(rng, 1, 90 if form == "decode" else 20)
    chunks = 0 if form == "decode" else _logu(rng, 1, 4)
    chunk = 0 if form == "decode" else _logu(rng, 2, 700)
    top = min(90e6 / (decode + chunks) / (kv * d), 2.0e9 / ((decode + chunks) * max(1, chunk) * heads), 60000)
    hi = _logu(rng, 30, max(31, top))
    return dict(case, decode=decode, chunks=chunks, chunk=chunk, lo=rng.randrange(0, hi + 1), hi=hi, alibi=rng.random() < 0.3)


# ---- what a case's numbers stand for --------------------------------------------------------------------------------

def _batch(case):
    """[(cached positions, new tokens)] of the sequences, in a fixed order; -1 new tokens: the request has just finished."""
    rng = random.Random(case["shape"])
    if case["kind"] == "packed":
        return [(0, rng.randint(case["lo"], case["hi"])) for _ in range(case["prompts"])]
    past = lambda: int(round(math.exp(rng.uniform(math.log(case["lo"] + 1), math.log(case["hi"] + 1))))) - 1
    seqs = [(past(), 1) for _ in range(case["decode"])]
    seqs += [(past(), rng.randint((case["chunk"] + 1) // 2, case["chunk"])) for _ in range(case["chunks"])]
    seqs += [(past(), -1) for _ in range(case.get("done", 0))]
    rng.shuffle(seqs)
    return seqs


def _rows(case):
    """Rows of the step's buffers: the new tokens and, behind them, rows that no sequence has."""
    return sum(max(q, 0) for _, q in _batch(case)) + case["pad"]


def _gen(seed, key):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 8191 + key)
    return g


def _qkv(case, seed):
    H, d, cols = case["heads"], case["d"], (case["heads"] + 2 * case["kv"]) * case["d"]
    x = torch.randn((_rows(case), cols), generator=_gen(seed, 1), device=DEVICE)
    x[:, :H * d] *= 2.0
    return x.to(DTYPES[case["dtype"]])


def _slopes(case):
    H = case["heads"]
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / H) for i in range(H)], dtype=torch.float32, device=DEVICE) if case.get("alibi") else None


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _offsets(case):
    cu = [0]
    for _, q in _batch(case):
        cu.append(cu[-1] + max(q, 0))
    return cu


def _pages(case, seed, spare):
    """(block table with each sequence's pages for `upto` of its positions, ids of the pool's pages behind those, pages in the pool).  A plan's sequences
    hold the pages of their cached positions, other kinds' those of their new tokens too; ids are in a random order."""
    P, batch = case["page"], _batch(case)
    upto = [past if case["kind"] == "plan" else past + max(q, 0) for past, q in batch]
    have = [-(-n // P) for n in upto]
    total = sum(-(-(past + max(q, 0)) // P) for past, q in batch) + spare
    ids = torch.randperm(total, generator=_gen(seed, 2), device=DEVICE).to(torch.int32)
    width = max(-(-(past + max(q, 0)) // P) for past, q in batch) + 1
    first = torch.tensor([sum(have[:i]) for i in range(len(have))], device=DEVICE)[:, None]
    j = torch.arange(width, device=DEVICE)[None, :]
    held = j < torch.tensor(have, device=DEVICE)[:, None]
    table = torch.where(held, ids[(first + j).clamp(max=total - 1)], torch.full_like(ids[:1], -1))
    return table.contiguous(), ids[sum(have):], total


def prepare(case, seed):
    kind, batch = case["kind"], _batch(case)
    s = {"case": case, "rows": _rows(case)}
    if kind == "plan":
        table, free, total = _pages(case, seed, 50)
        head = int(torch.randint(0, total, (1,), generator=_gen(seed, 3), device=DEVICE))
        ring = torch.full((total,), -1, dtype=torch.int32, device=DEVICE)
        ring[(head + torch.arange(free.numel(), device=DEVICE)) % total] = free
        n = len(batch)
        s.update(past=_ints([p for p, _ in batch]), q_lens=_ints([q for _, q in batch]), table=table, ring=ring, counters=_ints([head, free.numel()]))
        s["plan"] = tuple(torch.empty(m, dtype=torch.int32, device=DEVICE) for m in (n + 1, n, s["rows"], s["rows"], 2, 4))
        return s
    s["qkv"] = _qkv(case, seed)
    s["cu_q"] = _ints(_offsets(case))
    if kind != "append":
        s["slopes"] = _slopes(case)
        s["out"] = torch.zeros((s["rows"], case["heads"] * case["d"]), dtype=DTYPES[case["dtype"]], device=DEVICE)
        s["max_q"] = max(q for _, q in batch)
    if kind != "packed":
        P = case["page"]
        table, _, total = _pages(case, seed, 3)
        s["k"], s["v"] = (torch.randn((total, case["kv"], P, case["d"]), generator=_gen(seed, 4 + i), device=DEVICE).to(DTYPES[case["dtype"]]) for i in (0, 1))
        if kind == "paged":
            s.update(table=table, kv_lens=_ints([past + q for past, q in batch]), max_kv=max(past + q for past, q in batch))
        else:
            seq = torch.repeat_interleave(torch.arange(len(batch), device=DEVICE), torch.tensor([q for _, q in batch], device=DEVICE))
            pos = torch.arange(seq.numel(), device=DEVICE) - s["cu_q"][seq] + _ints([p for p, _ in batch])[seq]
            s["slots"] = torch.full((s["rows"],), -1, dtype=torch.int32, device=DEVICE)
            s["slots"][:seq.numel()] = (table[seq, pos // P] * P + pos % P).to(torch.int32)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        import paper_2403_01136_amd as lpq
        if kind == "plan":
            plan = lpq.lpq_paged_plan(s["past"], s["q_lens"], s["table"], s["ring"], s["counters"], case["page"], s["rows"], plan=s["plan"])
            return [*plan, s["table"], s["ring"]]
        if kind == "append":
            lpq.lpq_paged_append(s["qkv"], s["k"], s["v"], s["slots"])
            return [s["k"], s["v"]]
        if kind == "packed":
            return lpq.lpq_packed_attention(s["qkv"], s["cu_q"], case["heads"], case["kv"], max_q=s["max_q"], alibi_slopes=s["slopes"], out=s["out"])
        return lpq.lpq_paged_attention(s["qkv"], s["k"], s["v"], s["table"], s["cu_q"], s["kv_lens"], max_q=s["max_q"], max_kv=s["max_kv"],
                                       alibi_slopes=s["slopes"], out=s["out"])
    if kind == "plan":
        return _plain_plan(s)
    if kind == "append":
        return _plain_append(s)
    return _plain_attention(s)


def _plain_plan(s):
    """Prefix sums over the sequences, then every table entry, ring entry and row on its own."""
    P, M, n_pages = s["case"]["page"], s["rows"], s["ring"].numel()
    table, ring, past, q = s["table"], s["ring"].clone(), s["past"].long(), s["q_lens"].long()
    head, free = s["counters"].long()
    width, done, q = table.shape[1], q < 0, q.clamp(min=0)
    ends = torch.cumsum(q, 0)
    owned = ((past + P - 1) // P).clamp(max=width)
    late = (q > 0) & ((ends > M) | (past + q > width * P))                       # rows or table entries that are not there
    need = torch.where((q > 0) & ~late, (past + q + P - 1) // P - owned, torch.zeros_like(q))
    taken = torch.cumsum(need, 0)
    starved = late | ((need > 0) & (taken > free))
    given = torch.where(starved, torch.zeros_like(need), need)
    n_taken = torch.where(given > 0, taken, torch.zeros_like(taken)).max()
    back = torch.where(done, owned, torch.zeros_like(owned))
    n_back = torch.minimum(back.sum(), n_pages - free)
    # table entries of the new pages, ring entries of the returned ones
    j = torch.arange(width, device=DEVICE)[None, :]
    fresh = (j >= owned[:, None]) & (j < (owned + given)[:, None])
    source = (head + (taken - need)[:, None] + j - owned[:, None]) % n_pages
    new_table = torch.where(fresh, s["ring"][source], table)
    order = (torch.cumsum(back, 0) - back)[:, None] + j
    target = torch.where((j < back[:, None]) & (order < n_back), (head + free + order) % n_pages, torch.full_like(order, n_pages))
    ring = torch.cat([ring, ring[:1]]).scatter_(0, target.flatten(), table.flatten())[:n_pages]
    # rows
    r = torch.arange(M, device=DEVICE)
    seq = torch.searchsorted(ends, r, right=True).clamp(max=past.numel() - 1)
    served = (r < ends[-1]) & ~starved[seq]
    pos = past[seq] + r - (ends - q)[seq]
    page = new_table[seq, (pos // P).clamp(max=width - 1)].long()
    slots = torch.where(served & (page >= 0) & (page < n_pages), page * P + pos % P, torch.full_like(pos, -1))
    cu = torch.cat([ends[:1] * 0, ends]).clamp(max=M)
    kv = torch.where(done, torch.zeros_like(past), torch.where(starved, past, past + q))
    counters = torch.stack([(head + n_taken) % n_pages, free - n_taken + n_back])
    info = torch.stack([cu[-1], n_taken, n_back, starved.sum()])
    return [t.to(torch.int32) for t in (cu, kv, slots, torch.where(served, pos, torch.zeros_like(pos)), counters, info, new_table, ring)]


def _plain_append(s):
    """Every row's K and V put at their slot; a row without one repeats row 0, which has one."""
    case = s["case"]
    kv, d, P, H = case["kv"], case["d"], case["page"], case["heads"]
    rows = torch.where(s["slots"] >= 0, torch.arange(s["rows"], device=DEVICE), torch.zeros_like(s["slots"]))
    slots, new = s["slots"][rows].long(), s["qkv"][rows, H * d:].view(-1, 2, kv, d)
    at = ((slots // P)[:, None], torch.arange(kv, device=DEVICE)[None, :], (slots % P)[:, None])
    return [s["k"].index_put_(at, new[:, 0]), s["v"].index_put_(at, new[:, 1])]


def _plain_attention(s):
    """All sequences padded to the longest: scores, weights and their products in 32 bits."""
    case = s["case"]
    H, kv, d, M = case["heads"], case["kv"], case["d"], s["rows"]
    first, lens = s["cu_q"][:-1].long(), (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    t = torch.arange(s["max_q"], device=DEVICE)[None, :]
    live = t < lens[:, None]
    rows = torch.where(live, first[:, None] + t, torch.full_like(t, M))
    q = s["qkv"][rows.clamp(max=M - 1)][:, :, :H * d].float().view(*rows.shape, kv, H // kv, d)
    if case["kind"] == "packed":
        keys = s["qkv"][rows.clamp(max=M - 1)][:, :, H * d:].float().view(*rows.shape, 2, kv, d)
        k, v, ctx = keys[:, :, 0], keys[:, :, 1], lens
    else:
        P, ctx = case["page"], s["kv_lens"].long()
        j = torch.arange(s["max_kv"], device=DEVICE)
        page = s["table"][:, j // P].long().clamp(min=0)
        k, v = (pages[page, :, j % P].float() for pages in (s["k"], s["v"]))     # [sequence][position][head][d]
    n, L, G, T = k.shape[0], k.shape[1], H // kv, rows.shape[1]
    j = torch.arange(L, device=DEVICE)
    behind = j[None, None, :] - (ctx - lens)[:, None, None] - t[:, :, None]      # key position - query position
    hidden = ((behind > 0) | ~live[:, :, None])[:, None, None]
    sc = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(n, kv, G * T, d), k.permute(0, 2, 3, 1)).view(n, kv, G, T, L)
    sc *= 1.0 / math.sqrt(d)
    if s["slopes"] is not None:
        sc += s["slopes"].view(1, kv, G, 1, 1) * behind[:, None, None].float()
    sc.masked_fill_(hidden, float("-inf"))
    top = sc.amax(4, keepdim=True)
    sc.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = sc.sum(4, keepdim=True)
    o = torch.matmul(sc.view(n, kv, G * T, L), v.permute(0, 2, 1, 3)).view(n, kv, G, T, d) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 3, 1, 2, 4).reshape(n * T, H * d).to(s["out"].dtype)
    return torch.cat([s["out"], s["out"][:1]]).index_copy(0, rows.flatten(), o)[:M]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    batch = _batch(case)
    rows = sum(max(q, 0) for _, q in batch)
    if case["kind"] == "plan":
        P = case["page"]
        moved = sum(-(-(p + q) // P) - -(-p // P) if q > 0 else -(-p // P) if q < 0 else 0 for p, q in batch)
        return {"bytes": 16 * len(batch) + 8 * _rows(case) + 8 * moved + 36, "flops": 0}
    kv, d = case["kv"], case["d"]
    if case["kind"] == "append":
        return {"bytes": 8 * rows * kv * d + 4 * _rows(case), "flops": 0}
    pairs = sum(q * p + q * (q + 1) // 2 for p, q in batch)
    held = sum(p + q for p, q in batch)
    table = 4 * sum(-(-(p + q) // case["page"]) for p, q in batch) if case["kind"] == "paged" else 0
    return {"bytes": 4 * rows * case["heads"] * d + 4 * held * kv * d + 8 * len(batch) + table, "flops": 4 * pairs * case["heads"] * d}


# ---- the same from the definitions, in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    s, kind, batch = prepare(case, seed), case["kind"], _batch(case)
    if kind == "plan":
        return _exact_plan(s, batch)
    if kind == "append":
        return _exact_append(s, case)
    out = torch.zeros((s["rows"], case["heads"] * case["d"]), dtype=torch.float64, device=DEVICE)
    H, kv, d, slopes = case["heads"], case["kv"], case["d"], _slopes(case)
    for i, (past, q) in enumerate(batch):
        r0 = _offsets(case)[i]
        mine = s["qkv"][r0:r0 + q].double()
        if kind == "packed":
            k, v = (mine[:, (H + c * kv) * d:(H + (c + 1) * kv) * d].view(q, kv, d).transpose(0, 1) for c in (0, 1))
        else:
            ids = s["table"][i, :-(-(past + q) // case["page"])].long()
            k, v = (pages[ids].double().transpose(0, 1).reshape(kv, -1, d)[:, :past + q] for pages in (s["k"], s["v"]))
        j, p = torch.arange(past + q, device=DEVICE, dtype=torch.float64), torch.arange(past, past + q, device=DEVICE, dtype=torch.float64)
        for h in range(H):
            c = h // (H // kv)
            for t in range(0, q, 2048):
                e = min(t + 2048, q)
                logits = mine[t:e, h * d:(h + 1) * d] @ k[c].t() / math.sqrt(d)
                dist = j[None, :] - p[t:e, None]
                if slopes is not None:
                    logits = logits + float(slopes[h]) * dist
                out[r0 + t:r0 + e, h * d:(h + 1) * d] = torch.softmax(logits.masked_fill(dist > 0, float("-inf")), 1) @ v[c]
    return out


def _exact_plan(s, batch):
    """The step, one sequence, page and token after the other, on the host."""
    P, M = s["case"]["page"], s["rows"]
    table, ring, (head, free) = s["table"].tolist(), s["ring"].tolist(), s["counters"].tolist()
    width, n_pages = len(table[0]), len(ring)
    supply = [ring[(head + i) % n_pages] for i in range(free)]
    cu, kv, slots, positions = [0], [], [-1] * M, [0] * M
    rows = taken = wanted = starved = 0
    returned = []
    for i, (past, q) in enumerate(batch):
        if q < 0:
            returned += table[i][:min(-(-past // P), width)]
            kv.append(0)
            cu.append(min(rows, M))
            continue
        start, rows = rows, rows + q
        cu.append(min(rows, M))
        served = q == 0 or (rows <= M and past + q <= width * P)
        if served and q > 0:
            held, need = -(-past // P), -(-(past + q) // P) - -(-past // P)
            wanted += need
            served = need == 0 or wanted <= free
            if served and need:
                table[i][held:held + need] = supply[wanted - need:wanted]
                taken = wanted
            for t in range(q if served else 0):
                positions[start + t] = past + t
                slots[start + t] = table[i][(past + t) // P] * P + (past + t) % P
        starved += not served
        kv.append(past + q if served else past)
    returned = returned[:n_pages - free]
    for i, page in enumerate(returned):
        ring[(head + free + i) % n_pages] = page
    counters = [(head + taken) % n_pages, free - taken + len(returned)]
    return [_ints(x) for x in (cu, kv, slots, positions, counters, [cu[-1], taken, len(returned), starved], table, ring)]


def _exact_append(s, case):
    H, kv, d, P = case["heads"], case["kv"], case["d"], case["page"]
    k, v = s["k"].double(), s["v"].double()
    for r, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            row = s["qkv"][r, H * d:].double().view(2, kv, d)
            k[slot // P, :, slot % P], v[slot // P, :, slot % P] = row[0], row[1]
    return [k, v]
