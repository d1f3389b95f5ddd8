"""The compacted cache held in 4 bits and in pages, as timed cases of five operators.

  append   rows of K and V (a prompt's kept rows, or the new row of every sequence) are rounded to 4 bits and put behind
           the rows that their heads have, in pages taken from a pool; a last page that others share is copied first
  read     rows of the cache as bf16, packed head by head: what the library's other stages take
  attend   one decoding step of every sequence on its cache
  fork     every sequence takes over another's pages (a beam's parent), its own cut short, or none
  keep     every head keeps given rows, moved together; the pages that it no longer needs are free

A row of d channels is d / 32 blocks. A block stands for code * 2^(e - 127): one byte e and 32 codes of four bits, a sign
and one of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6. e is the smallest with max|x| <= 7 * 2^(e - 127), within 2 and 252
(2 for a block of zeros); a value goes to the nearest magnitude, in the middle to the even code, beyond 6 to 6. A block
with an infinity or NaN has e = 255, codes 0, and stands for NaN. A page of P rows of one KV head is K's codes [P][d / 2]
(even channel in the low half of a byte), V's codes, K's e [P][d / 32], V's e.

State: table [heads][entries] of page numbers, lengths [heads], refs [pages] (how many heads have the page), state [2]: how
many pages are free (refs 0), and where the search for free ones begins. It goes upwards from there and round.

A case is a dict of plain values. Common: do, q_heads, kv_heads, dim, page (rows). Lists of sizes are drawn from
`sizes_seed`, spread over their logarithm, so that a case stays plain. seqs may be (sequence, layer) pairs.
"""
import math
import random

import numpy as np
import torch

own = False

# query heads, KV heads, head_dim: the geometries of this repository's workloads and tests
GEOMETRIES = [(28, 4, 128), (32, 4, 128), (8, 2, 256), (8, 2, 64)]
KEPT = 0.4          # share of a prompt's tokens that its eviction kept


def _case(name, do, geometry, page, seqs, fewest, most, sizes_seed=0, **more):
    """fewest, most: rows of a head before the call (append of prompts: tokens of a prompt)."""
    return {"name": name, "do": do, "q_heads": geometry[0], "kv_heads": geometry[1], "dim": geometry[2], "page": page,
            "seqs": seqs, "fewest": fewest, "most": most, "sizes_seed": sizes_seed, **more}


def listed():
    return [
        # the new row of 48 sequences in generation, every third the fork of the one before it: a launch or two
        _case("append_step_48", "append", (28, 4, 128), 64, 48, 200, 3000, 1, new=1, forked=3, evicted=False, layout="head"),
        # a prompt of 28 layers after its eviction: kept rows, a budget for each head, into an empty cache
        _case("append_28x8192_kept", "append", (28, 4, 128), 64, 28, 8192, 8192, 2, new=0, forked=0, evicted=True, layout="head"),
        # one sequence back to bf16, for the scoring of its rows
        _case("read_1x8192", "read", (28, 4, 128), 64, 1, 8192, 8192),
        # ragged sequences of wide heads
        _case("read_16xragged_d256", "read", (8, 2, 256), 128, 16, 500, 20000, 3),
        # one sequence on what a short prompt kept: the smallest step, where latency counts
        _case("attend_1x900", "attend", (28, 4, 128), 64, 1, 500, 900, 4, lse=False),
        # a serving batch, each head with a budget of its own
        _case("attend_16xragged", "attend", (32, 4, 128), 64, 16, 300, 13000, 5, lse=False),
        # wide heads, the log-sum-exp for a second part of the cache
        _case("attend_6xragged_d256", "attend", (8, 2, 256), 128, 6, 1000, 20000, 6, lse=True),
        # a large batch of long sequences
        _case("attend_64x32768", "attend", (28, 4, 128), 64, 64, 32768, 32768, lse=False),
        # a beam of four goes on from two of its members
        _case("fork_4_of_1000", "fork", (28, 4, 128), 64, 4, 700, 1000, 7, drop=0, gone=0),
        # a batch of samples: a third take over others, some end, all lose up to seven rejected rows
        _case("fork_64_of_13107", "fork", (28, 4, 128), 64, 64, 6000, 13107, 8, drop=7, gone=8),
        # caches that grew are brought back to a budget
        _case("keep_4_of_1100", "keep", (28, 4, 128), 64, 4, 1000, 1100, 9, share=0.9),
        # long caches are halved
        _case("keep_16_of_8192", "keep", (32, 4, 128), 64, 16, 8192, 8192, 10, share=0.5),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    geometry = rng.choice(GEOMETRIES)
    heads, d = geometry[1], geometry[2]
    do = rng.choice(["append", "read", "attend", "attend", "fork", "keep"])
    seed, page = rng.randrange(1 << 20), rng.choice([32, 64, 128, 256])
    if do == "append":
        if rng.random() < 0.5:
            case = _case("", do, geometry, page, _spread(rng, 1, 64), 1, _spread(rng, 1, 4000), seed,
                         new=rng.choice([1, 1, rng.randint(2, 40)]), forked=rng.choice([0, 2, 5]), evicted=False,
                         layout=rng.choice(["head", "token"]))
        else:
            most = _spread(rng, 10, 32768)
            seqs = max(1, min(_spread(rng, 1, 28), int(1.1e8 / (most * heads * d))))
            case = _case("", do, geometry, page, seqs, max(1, most // rng.choice([1, 4, 20])), most, seed, new=0, forked=0,
                         evicted=rng.random() < 0.7, layout=rng.choice(["head", "token"]))
    elif do == "attend":
        most = _spread(rng, 1, 32768)
        seqs = max(1, min(_spread(rng, 1, 64), int(1.07e9 / (most * heads * d))))
        case = _case("", do, geometry, page, seqs, max(1, most // rng.choice([1, 4, 40])), most, seed, lse=rng.random() < 0.5)
    else:
        most = _spread(rng, 3, 20000)
        seqs = max(1, min(_spread(rng, 1, 64), int(6e7 / (most * heads * d))))
        more = ({"drop": rng.choice([0, 0, 9]), "gone": rng.choice([0, 0, seqs // 4])} if do == "fork" else
                {"share": rng.choice([0.3, 0.7, 0.97])} if do == "keep" else {})
        case = _case("", do, geometry, page, seqs, max(1, most // rng.choice([1, 4, 20])), most, seed, **more)
    del case["name"]
    return case


# ---- sizes ---------------------------------------------------------------------------------------------------------

def _pages_of(rows, P):
    return -(-rows // P)


def _rows_before(case):
    """Rows of every head before the call."""
    r = random.Random(case["sizes_seed"])
    H = case["kv_heads"]
    if case["do"] == "append" and not case["new"]:
        return [0] * (case["seqs"] * H)
    out = []
    for x in range(case["seqs"]):
        n = _spread(r, case["fewest"], case["most"]) if x and case["fewest"] < case["most"] else case["most"]
        forked = case["do"] == "append" and case["forked"] and x % case["forked"] == case["forked"] - 1
        # heads of a sequence have budgets of their own, and have grown by as many rows since
        rows = [n if h == 0 or case["fewest"] == case["most"] else max(1, int(n * r.uniform(0.4, 1))) for h in range(H)]
        out += out[-H:] if forked and out else rows
    return out


def _rows_added(case):
    """append: tokens of every item, and rows that each of its heads gets."""
    r = random.Random(case["sizes_seed"] + 1)
    H = case["kv_heads"]
    if case["new"]:
        lens = [case["new"]] * case["seqs"]
        return lens, [case["new"]] * (case["seqs"] * H)
    lens = [_spread(r, case["fewest"], case["most"]) if x and case["fewest"] < case["most"] else case["most"] for x in range(case["seqs"])]
    if not case["evicted"]:
        return lens, [L for L in lens for _ in range(H)]
    added = []
    for L in lens:
        share = [r.uniform(0.4, 1.6) for _ in range(H)]
        added += [max(1, min(L, int(L * KEPT * H * s / sum(share)))) for s in share]
    return lens, added


def _rows_kept(case):
    r = random.Random(case["sizes_seed"] + 1)
    return [max(1, min(n, int(n * case["share"] * r.uniform(0.8, 1.2)))) for n in _rows_before(case)]


def _read_from(case, before):
    """append: the first row that is read back, that of the page which the call writes first."""
    return [n // case["page"] * case["page"] for n in before]


def work(case):
    H, Hq, d, P = case["kv_heads"], case["q_heads"], case["dim"], case["page"]
    held = d * 17 // 16                       # bytes of a row of K and V, codes and scales
    before = _rows_before(case)
    if case["do"] == "append":
        _, added = _rows_added(case)
        back = sum(n + a - f for n, a, f in zip(before, added, _read_from(case, before)))
        return {"bytes": sum(added) * (4 * d + held + (4 if case["evicted"] else 0)) + back * (held + 4 * d),
                "flops": sum(added) * d * 6 + back * d * 2}
    if case["do"] == "read":
        return {"bytes": sum(before) * (held + 4 * d), "flops": sum(before) * d * 2}
    if case["do"] == "attend":
        return {"bytes": sum(before) * held + case["seqs"] * Hq * (4 * d + (4 if case["lse"] else 0)),
                "flops": 4 * (Hq // H) * d * sum(before)}
    if case["do"] == "fork":
        # every entry read and written, and the count of its page
        entries = sum(_pages_of(n, P) for n in before)
        return {"bytes": entries * 16, "flops": entries}
    kept = sum(_rows_kept(case))
    return {"bytes": kept * (2 * held + 4) + kept * (held + 4 * d), "flops": kept * d * 2}


# ---- the format ----------------------------------------------------------------------------------------------------

def _encode(x):
    """[..., d] in any type -> codes uint8 [..., d / 2], scales uint8 [..., d / 32]."""
    x = x.float().unflatten(-1, (-1, 32))
    a = x.abs().amax(-1)
    fine = torch.isfinite(a)
    m, e = torch.frexp(torch.where(fine, a, 0.0))                       # a = m * 2^e, m in [0.5, 1)
    k = torch.where(a == 0, -125, (e - 3 + (m > 0.875)).clamp(-125, 125))
    y = torch.ldexp(torch.where(fine[..., None], x, 0.0), -k[..., None])
    z = y.abs()
    code = ((z > 0.25).to(torch.uint8) + (z >= 0.75) + (z > 1.25) + (z >= 1.75) + (z > 2.5) + (z >= 3.5) + (z > 5)
            + torch.signbit(y).to(torch.uint8) * 8)
    code = torch.where(fine[..., None], code, 0).flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | code[..., 1] << 4, torch.where(fine, k + 127, 255).to(torch.uint8)


def _decode(codes, scales):
    """The values that codes and scales stand for, in 32 bits."""
    magnitude = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).unflatten(-1, (-1, 32))
    scale = torch.where(scales == 255, math.nan, torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127))
    return (magnitude[code.int()] * scale[..., None]).flatten(-2)


def _sections(pool, P, d):
    """Views of a pool [pages, bytes]: K's codes, V's codes, K's scales, V's scales, each [pages, P, ...]."""
    at = [0, P * d // 2, P * d, P * d + P * d // 32, P * d + P * d // 16]
    return [pool[:, a:b].unflatten(1, (P, -1)) for a, b in zip(at, at[1:])]


# ---- inputs --------------------------------------------------------------------------------------------------------

def _gen(seed, part):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 16 + part)


def _rows(shape, gen, keys=False):
    """bf16 rows; keys have a part in common, and one token in 64 that stands out."""
    x = torch.randn(shape, generator=gen, device="cuda")
    if keys:
        x += 0.5 * torch.randn(shape[-1], generator=gen, device="cuda")
        x *= 1 + (torch.rand((*shape[:-1], 1), generator=gen, device="cuda") < 1 / 64)
    return x.to(torch.bfloat16)


def _cu(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    H, Hq, d, P, n_seqs = case["kv_heads"], case["q_heads"], case["dim"], case["page"], case["seqs"]
    before, do = _rows_before(case), case["do"]
    heads = len(before)
    s = {"case": case, "before": before}
    after = before
    if do == "append":
        s["lens"], s["added"] = _rows_added(case)
        after = [n + a for n, a in zip(before, s["added"])]
    width = max(_pages_of(n, P) for n in after) + 1
    spare = sum(_pages_of(a, P) + 1 for a in after) if do in ("append", "keep") else heads
    n_pages = sum(_pages_of(n, P) for n in before) + spare + 7
    # a pool in use for a while: a head's pages lie anywhere in it
    gen = _gen(seed, 0)
    anywhere = torch.randperm(n_pages, generator=gen, device="cuda").int()
    lengths = _int(before)
    mine = torch.arange(width, device="cuda") < _pages_of_each(lengths, P)[:, None]
    table = torch.where(mine, anywhere[(mine.flatten().cumsum(0) - 1).view(mine.shape).clamp_min(0)], -1)
    if do == "append" and case["forked"]:
        for x in range(case["forked"] - 1, n_seqs, case["forked"]):     # a sequence that has the pages of the one before it
            table[x * H:(x + 1) * H] = table[(x - 1) * H:x * H]
    if do == "fork":
        r = random.Random(case["sizes_seed"] + 2)
        parents = list(range(n_seqs))
        for x in r.sample(range(n_seqs), max(1, n_seqs // 3)):
            parents[x] = r.randrange(n_seqs)
        for x in r.sample(range(n_seqs), case["gone"]):
            parents[x] = -1
        s["parents"] = _int(parents)
        s["drop"] = _int([r.randint(0, case["drop"]) for _ in range(n_seqs)]) if case["drop"] else None
        s["parent_list"] = parents
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs.index_add_(0, table.flatten().clamp_min(0), mine.flatten().int())
    state = torch.stack(((refs == 0).sum(), torch.randint(n_pages, (), generator=gen, device="cuda"))).int()
    # one buffer, so that one copy takes a pass back to where it began
    s["begin"] = torch.cat((table.flatten().int(), lengths, refs, state))
    s["live"], s["n_pages"], s["width"] = s["begin"].clone(), n_pages, width
    # (a page more than the pool has: where the plain form's masked stores go)
    s["pool"] = torch.empty((n_pages + 1, P * d * 17 // 16), dtype=torch.uint8, device="cuda")
    if do == "append":
        s["pool"].random_(0, 240, generator=_gen(seed, 1))              # (no scale says NaN)
    elif do != "fork":
        gk, gv = _gen(seed, 1), _gen(seed, 2)
        step = max(1, (1 << 26) // (P * d))
        for a in range(0, n_pages + 1, step):
            kc, vc, ks, vs = _sections(s["pool"][a:a + step], P, d)
            for codes, scales, g, keys in ((kc, ks, gk, True), (vc, vs, gv, False)):
                c, e = _encode(_rows((*codes.shape[:2], d), g, keys))
                codes.copy_(c)
                scales.copy_(e)
    if do == "append":
        shape = (sum(s["lens"]) * H, d)
        s["k"], s["v"] = _rows(shape, _gen(seed, 3), keys=True), _rows(shape, _gen(seed, 4))
        s["cu"] = _cu(s["lens"])
        # items come in another order than their sequences
        order = random.Random(case["sizes_seed"] + 3).sample(range(n_seqs), n_seqs)
        s["order"], s["seqs"] = order, _int(order)
        s["before"] = before = [before[x * H + h] for x in order for h in range(H)]       # by item
        first = _read_from(case, before)
        back = [0] * heads
        s["first_list"] = [0] * heads
        for i, x in enumerate(order):
            for h in range(H):
                back[x * H + h] = before[i * H + h] + s["added"][i * H + h] - first[i * H + h]
                s["first_list"][x * H + h] = first[i * H + h]
        s["first"], s["cu_rows"], s["total"] = _int(s["first_list"]), _cu(back), sum(back)
        if case["evicted"]:
            r = np.random.default_rng(case["sizes_seed"] * 1000 + seed)
            L = np.repeat(s["lens"], H)
            s["index_list"] = [np.sort(r.choice(n, a, replace=False)) for n, a in zip(L, s["added"])]
            s["indices"], s["cu_b"] = _int(np.concatenate(s["index_list"])), _cu(s["added"])
    elif do == "read":
        s["cu_rows"], s["total"] = _cu(before), sum(before)
    elif do == "attend":
        s["q"] = _rows((n_seqs, Hq, d), _gen(seed, 3)) * 1.5
    elif do == "keep":
        r = np.random.default_rng(case["sizes_seed"] * 1000 + seed)
        kept = _rows_kept(case)
        # the first rows stay more often than not: a prompt's beginning
        s["index_list"] = [np.sort(np.argsort(r.random(n) + (np.arange(n) >= n // 4))[:b]) for n, b in zip(before, kept)]
        s["indices"], s["cu_b"], s["total"] = _int(np.concatenate(s["index_list"])), _cu(kept), sum(kept)
    return s


def _pages_of_each(rows, P):
    return torch.div(rows + P - 1, P, rounding_mode="floor")


def _parts(s):
    """table, lengths, refs and state in the buffer that holds all four."""
    heads = s["case"]["seqs"] * s["case"]["kv_heads"]
    a = heads * s["width"]
    b = a + heads
    c = b + s["n_pages"]
    live = s["live"]
    return live[:a].view(heads, -1), live[a:b], live[b:c], live[c:]


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _free_pages(refs, state):
    """Page numbers in the order in which they are taken (only those that are free count)."""
    n = refs.numel()
    order = (torch.arange(n, device=refs.device) + state[1]) % n
    free = refs[order] == 0
    by_rank = torch.zeros(n + 1, dtype=torch.long, device=refs.device)
    return by_rank.scatter_(0, torch.where(free, free.cumsum(0) - 1, n), order)


def _take(refs, state, pages, taken, given_back):
    """refs and state after the first `taken` of `pages` went to heads, and heads gave back `given_back` = (pages, counts)."""
    n = refs.numel()
    refs.index_add_(0, pages[:n], (torch.arange(n, device=refs.device) < taken).int())
    refs.index_add_(0, given_back[0].clamp_min(0).flatten().long(), -given_back[1].flatten().int())
    state[1] = torch.where(taken > 0, (pages[(taken - 1).clamp_min(0)] + 1) % n, state[1])
    state[0] = (refs == 0).sum()


def _read(s, table, first, cu_rows, total):
    P, d = s["case"]["page"], s["case"]["dim"]
    r = torch.arange(total, device=table.device)
    g = torch.searchsorted(cu_rows, r.int(), right=True) - 1
    at = r - cu_rows[g] + (0 if first is None else first[g])
    page, row = table[g, at // P].long(), at % P
    kc, vc, ks, vs = (x[page, row] for x in _sections(s["pool"], P, d))
    return _decode(kc, ks).to(torch.bfloat16), _decode(vc, vs).to(torch.bfloat16)


def _plain_append(s):
    case = s["case"]
    H, d, P = case["kv_heads"], case["dim"], case["page"]
    s["live"].copy_(s["begin"])
    table, lengths, refs, state = _parts(s)
    dev = table.device
    items, nowhere = len(s["lens"]), s["n_pages"]
    L = (s["cu"][1:] - s["cu"][:-1]).repeat_interleave(H)
    cu = s["cu_b"].long() if case["evicted"] else torch.nn.functional.pad(L.long().cumsum(0), (1, 0))
    count = cu[1:] - cu[:-1]
    head = (s["seqs"].long()[:, None] * H + torch.arange(H, device=dev)).flatten()
    start = lengths[head].long()
    end = start + count
    old = table[head]
    last = old.gather(1, (start // P)[:, None]).squeeze(1).long()       # the page that the first row goes to, if it is there
    copy = (start % P != 0) & (count > 0) & (refs[last.clamp_min(0)] > 1)
    first_new = _pages_of_each(start, P) - copy.long()
    need = _pages_of_each(end, P) - first_new
    pages, pre = _free_pages(refs, state), need.cumsum(0) - need
    j = torch.arange(s["width"], device=dev)
    fresh = (j >= first_new[:, None]) & (j < (first_new + need)[:, None])
    new = torch.where(fresh, pages[(pre[:, None] + j - first_new[:, None]).clamp(0, nowhere)], old.long())
    # shared last pages
    onto = new.gather(1, (start // P)[:, None]).squeeze(1)
    s["pool"][torch.where(copy, onto, nowhere)] = s["pool"][last.clamp_min(0)]
    # rows
    r = torch.arange(sum(s["added"]), device=dev)
    g = torch.searchsorted(cu, r, right=True) - 1
    t = r - cu[g]
    token = s["indices"].long() if case["evicted"] else t
    item, h = g // H, g % H
    base = s["cu"].long()[item]
    src = (base + token) * H + h if case["layout"] == "token" else base * H + h * L[g] + token
    at = start[g] + t
    page, row = new[g, at // P], at % P
    kc, vc, ks, vs = _sections(s["pool"], P, d)
    kc[page, row], ks[page, row] = _encode(s["k"][src])
    vc[page, row], vs[page, row] = _encode(s["v"][src])
    table[head] = new.int()
    lengths[head] = end.int()
    _take(refs, state, pages, need.sum(), (last, copy))
    return *_read(s, table, s["first"], s["cu_rows"], s["total"]), table, lengths, refs, state


def _plain_attend(s):
    case = s["case"]
    H, Hq, d, P = case["kv_heads"], case["q_heads"], case["dim"], case["page"]
    table, lengths, _, _ = _parts(s)
    n, most = table.shape[0], max(s["before"])
    page = table[:, :_pages_of(most, P)].clamp_min(0).long()
    kc, vc, ks, vs = _sections(s["pool"], P, d)
    there = torch.arange(page.shape[1] * P, device=page.device) < lengths[:, None]
    q = s["q"].float().view(n, Hq // H, d)
    z = torch.bmm(q, _decode(kc[page], ks[page]).view(n, -1, d).transpose(1, 2).contiguous())
    z = z.mul_(1 / math.sqrt(d)).masked_fill_(~there[:, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    p = z.sub_(m).exp_()
    den = p.sum(-1, keepdim=True)
    out = torch.bmm(p, _decode(vc[page], vs[page]).view(n, -1, d).masked_fill_(~there[:, :, None], 0)) / den
    out = out.view(-1, Hq, d).to(torch.bfloat16)
    return (out, (m + den.log()).view(-1, Hq)) if case["lse"] else out


def _plain_fork(s):
    case = s["case"]
    H, P = case["kv_heads"], case["page"]
    s["live"].copy_(s["begin"])
    table, lengths, refs, state = _parts(s)
    dev = table.device
    parent = s["parents"].long().repeat_interleave(H)
    src = parent.clamp_min(0) * H + torch.arange(H, device=dev).repeat(case["seqs"])
    rows = lengths[src] - (0 if s["drop"] is None else s["drop"].repeat_interleave(H))
    rows = torch.where(parent < 0, 0, rows.clamp_min(0))
    j = torch.arange(s["width"], device=dev)
    has, had = j < _pages_of_each(rows, P)[:, None], j < _pages_of_each(lengths, P)[:, None]
    new = torch.where(has, table[src], table)
    refs.index_add_(0, new.clamp_min(0).flatten(), has.flatten().int())
    refs.index_add_(0, table.clamp_min(0).flatten(), -had.flatten().int())
    table.copy_(new)
    lengths.copy_(rows)
    state[0] = (refs == 0).sum()
    return table, lengths, refs, state


def _plain_keep(s):
    case = s["case"]
    P, d, nowhere = case["page"], case["dim"], s["n_pages"]
    s["live"].copy_(s["begin"])
    table, lengths, refs, state = _parts(s)
    dev, old = table.device, table.long()
    cu = s["cu_b"].long()
    b, rows = cu[1:] - cu[:-1], lengths.long()
    cut = b < rows
    j = torch.arange(s["width"], device=dev)
    # whole pages that stay as they are: rows are in order, so that the last one says it for all
    last = (j + 1) * P - 1
    whole = (last < b[:, None]) & (s["indices"][(cu[:-1, None] + last).clamp_max(s["total"] - 1)] == last)
    same = whole.int().cumprod(1).sum(1)
    need = torch.where(cut, _pages_of_each(b, P) - same, 0)
    pages, pre = _free_pages(refs, state), need.cumsum(0) - need
    fresh = (j >= same[:, None]) & (j < (same + need)[:, None])
    new = torch.where(fresh, pages[(pre[:, None] + j - same[:, None]).clamp(0, nowhere)], old)
    r = torch.arange(s["total"], device=dev)
    g = torch.searchsorted(cu, r, right=True) - 1
    t, at = r - cu[g], s["indices"].long()
    moves = cut[g] & (t >= same[g] * P)
    onto, page = torch.where(moves, new[g, t // P], nowhere), old[g, at // P].clamp_min(0)
    for x in _sections(s["pool"], P, d):
        x[onto, t % P] = x[page, at % P]
    gone = cut[:, None] & (j >= same[:, None]) & (j < _pages_of_each(rows, P)[:, None])
    table.copy_(new)
    lengths.copy_(torch.minimum(b, rows))
    _take(refs, state, pages, need.sum(), (old, gone))
    return *_read(s, table, None, s["cu_b"], s["total"]), table, lengths, refs, state


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    do = state["case"]["do"]
    if own:
        return _own(state)
    if do == "read":
        return _read(state, _parts(state)[0], None, state["cu_rows"], state["total"])
    return {"append": _plain_append, "attend": _plain_attend, "fork": _plain_fork, "keep": _plain_keep}[do](state)


def _own_setup(s):
    """What a program lays out once: the cache, its outputs and a workspace."""
    import paper_2604_06694_amd as A
    case, do = s["case"], s["case"]["do"]
    p = A.Params(case["q_heads"], case["kv_heads"], case["dim"], 0,
                 kv_layout=A.LAYOUT_TOKEN_MAJOR if case.get("layout") == "token" else A.LAYOUT_HEAD_MAJOR)
    table, lengths, refs, state = _parts(s)
    pages = A.Pages(s["pool"][:s["n_pages"]].flatten(), table, lengths, refs, state, case["page"])
    size = {"append": lambda: A.pages_append_workspace_bytes(p, pages, len(s["lens"]), sum(s["added"])),
            "read": lambda: 0, "attend": lambda: A.pages_attend_workspace_bytes(p, pages),
            "fork": lambda: A.pages_fork_workspace_bytes(p, pages),
            "keep": lambda: A.pages_keep_workspace_bytes(p, pages, s["total"])}[do]()
    s["A"], s["p"], s["pages"] = A, p, pages
    s["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device="cuda")
    if do == "attend":
        s["out"] = torch.empty_like(s["q"])
        s["out_lse"] = torch.empty(s["q"].shape[:2], device="cuda") if case["lse"] else None
    elif do != "fork":
        s["k_back"] = torch.empty((s["total"], case["dim"]), dtype=torch.bfloat16, device="cuda")
        s["v_back"] = torch.empty_like(s["k_back"])


def _own(s):
    if "A" not in s:
        _own_setup(s)
    A, p, pages, do = s["A"], s["p"], s["pages"], s["case"]["do"]
    if do == "read":
        return A.pages_read(p, pages, s["cu_rows"], s["total"], k_out=s["k_back"], v_out=s["v_back"])
    if do == "attend":
        out = A.pages_attend(p, pages, s["q"], out=s["out"], lse=s["out_lse"], workspace=s["ws"])
        return (out, s["out_lse"]) if s["case"]["lse"] else out
    s["live"].copy_(s["begin"])
    state = pages.table, pages.lengths, pages.refs, pages.state
    if do == "fork":
        A.pages_fork(p, pages, s["parents"], drop=s["drop"], workspace=s["ws"])
        return state
    if do == "append":
        A.pages_append(p, pages, s["k"], s["v"], s["lens"], indices=s.get("indices"), cu_budgets=s.get("cu_b"),
                       total_rows=sum(s["added"]), seqs=s["seqs"], cu_seqlens=s["cu"], workspace=s["ws"])
        return *A.pages_read(p, pages, s["cu_rows"], s["total"], first=s["first"], k_out=s["k_back"], v_out=s["v_back"]), *state
    A.pages_keep(p, pages, s["indices"], s["cu_b"], s["total"], workspace=s["ws"])
    return *A.pages_read(p, pages, s["cu_b"], s["total"], k_out=s["k_back"], v_out=s["v_back"]), *state


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------

def _rounded(x):
    """What 4 bits hold of x [rows, d]."""
    x = x.double().view(x.shape[0], -1, 32)
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.where(top > 0, torch.ceil(torch.log2(top / 7)), -125).clamp(-125, 125))
    y = x / scale
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    return ((y / step).round() * step).clamp(-6, 6).mul(scale).flatten(1)


def _held(s, page, row, keys):
    """The values in rows of pages, in 64 bits."""
    P, d = s["case"]["page"], s["case"]["dim"]
    at, half = page.long() * (P * d * 17 // 16), P * d // 2
    flat = s["pool"].flatten()
    c = torch.arange(d, device="cuda")
    code = flat[(at + (0 if keys else half) + row * (d // 2))[:, None] + c // 2].long() >> (c % 2 * 4) & 15
    e = flat[(at + 2 * half + (0 if keys else P * d // 32) + row * (d // 32))[:, None] + c // 32].double()
    size = code % 8
    value = torch.where(size < 2, size / 2, (1 + size % 2 / 2).double() * torch.exp2((size // 2 - 1).double()))
    return torch.where(code >= 8, -value, value).double() * torch.exp2(e - 127)


def _search(refs, at, n):
    found = []
    for i in range(len(refs)):
        if len(found) == n:
            break
        page = (at + i) % len(refs)
        if refs[page] == 0:
            found.append(page)
    return found


def exact(case, seed):
    s = prepare(case, seed)
    H, Hq, d, P = case["kv_heads"], case["q_heads"], case["dim"], case["page"]
    table, lengths, refs, state = (x.cpu().numpy().copy() for x in _parts(s))
    heads = case["seqs"] * H

    def held(g, at, keys, rows):
        rows = torch.as_tensor(np.asarray(rows), device="cuda")
        return _held(s, torch.as_tensor(at[g], device="cuda")[rows // P], rows % P, keys)

    if case["do"] == "read":
        return tuple(torch.cat([held(g, table, keys, np.arange(s["before"][g])) for g in range(heads)]) for keys in (True, False))
    if case["do"] == "attend":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
        for g in range(heads):
            x, h = divmod(g, H)
            mine = slice(h * (Hq // H), (h + 1) * (Hq // H))
            rows = np.arange(s["before"][g])
            z = s["q"][x, mine].double() @ held(g, table, True, rows).T.contiguous() / math.sqrt(d)
            lse[x, mine] = torch.logsumexp(z, 1)
            out[x, mine] = torch.softmax(z, 1) @ held(g, table, False, rows)
        return (out, lse) if case["lse"] else out
    begun = table.copy()
    if case["do"] == "fork":
        drop = [0] * case["seqs"] if s["drop"] is None else s["drop"].tolist()
        rows_then = lengths.copy()
        for x, parent in enumerate(s["parent_list"]):
            for h in range(H):
                g = x * H + h
                for j in range(_pages_of(int(rows_then[g]), P)):
                    refs[begun[g, j]] -= 1
                n = 0 if parent < 0 else max(0, int(rows_then[parent * H + h]) - drop[x])
                for j in range(_pages_of(n, P)):
                    table[g, j] = begun[parent * H + h, j]
                    refs[table[g, j]] += 1
                lengths[g] = n
        state[0] = int((refs == 0).sum())
        return table, lengths, refs, state
    free, taken, released = refs.copy(), 0, []
    plan = _search(refs, int(state[1]), int(state[0]))
    back = [[None] * heads, [None] * heads]
    if case["do"] == "append":
        starts = np.concatenate([[0], np.cumsum(s["lens"])])
        for i, x in enumerate(s["order"]):
            for h in range(H):
                a, g = i * H + h, x * H + h
                n, added, L = int(lengths[g]), s["added"][a], s["lens"][i]
                first = -(-n // P)
                if n % P and free[table[g, n // P]] > 1:
                    released.append(table[g, n // P])
                    first -= 1
                for j in range(first, _pages_of(n + added, P)):
                    table[g, j] = plan[taken]
                    taken += 1
                lengths[g] = n + added
                token = torch.as_tensor(s["index_list"][a] if case["evicted"] else np.arange(added), device="cuda")
                src = (int(starts[i]) + token) * H + h if case["layout"] == "token" else int(starts[i]) * H + h * L + token
                for which, (x_in, keys) in enumerate(((s["k"], True), (s["v"], False))):
                    kept = held(g, begun, keys, np.arange(s["first_list"][g], n)) if n > s["first_list"][g] else torch.empty((0, d), device="cuda").double()
                    back[which][g] = torch.cat((kept, _rounded(x_in[src])))
    else:
        for g in range(heads):
            index, n = s["index_list"][g], int(lengths[g])
            if len(index) >= n:
                for which, keys in enumerate((True, False)):
                    back[which][g] = held(g, begun, keys, index)
                continue
            same = 0
            while (same + 1) * P <= len(index) and index[(same + 1) * P - 1] == (same + 1) * P - 1:
                same += 1
            released += list(begun[g, same:_pages_of(n, P)])
            for j in range(same, _pages_of(len(index), P)):
                table[g, j] = plan[taken]
                taken += 1
            lengths[g] = len(index)
            for which, keys in enumerate((True, False)):
                back[which][g] = held(g, begun, keys, index)
    for page in plan[:taken]:
        refs[page] += 1
    for page in released:
        refs[page] -= 1
    if taken:
        state[1] = (plan[taken - 1] + 1) % len(refs)
    state[0] = int((refs == 0).sum())
    return torch.cat(back[0]), torch.cat(back[1]), table, lengths, refs, state
