"""What surrounds one prefill's eviction in a generating program, as timed cases of three operators.

  accumulate         the attention weight that every cached token has received from ALL queries of a prompt (or of one
                     chunk of it), added to a running total: what an eviction by accumulated weight ranks tokens by
  decode_shared      one decoding step of sequences that share the compacted cache of a prompt (samples, beams, requests
                     with one recording) and own the rows that they have generated since; the step appends its own row
                     and adds the weights that the own rows received to their totals
  evict_accumulated  own rows beyond a budget go: the most recent stay, then those of the largest accumulated weight; the
                     slots of the others take the kept rows from the end of the cache, in place

A case is a dict of plain values. Common: do, q_heads, kv_heads, dim. Lists of sizes are drawn from `sizes_seed` between
two ends (spread over their logarithm), so that a case stays plain.
"""
import math
import random

import numpy as np
import torch

own = False

# query heads, KV heads, head_dim: the geometries of this repository's workloads and tests
GEOMETRIES = [(28, 4, 128), (32, 4, 128), (8, 2, 256), (8, 2, 64)]
KEPT = 0.4          # share of a prompt's tokens that its eviction kept


def _accumulate(name, geometry, items, shortest, longest=None, queries=0, layout="head", lse=False, sizes_seed=0):
    """queries: of the newest chunk of each prompt (0: the whole prompt). layout: head ([H][L][d] per item), token
    ([L][H][d]) or slab (a padded [items][H][L_max][d] cache, totals [items][H][L_max])."""
    return {"name": name, "do": "accumulate", "q_heads": geometry[0], "kv_heads": geometry[1], "dim": geometry[2],
            "items": items, "shortest": shortest, "longest": longest or shortest, "queries": queries,
            "layout": layout, "lse": lse, "sizes_seed": sizes_seed}


def _step(name, geometry, prompts, prompt, sharing, rows, capacity, fewest=None, weights=True, sizes_seed=0):
    """prompts (0: no shared part, `sharing` sequences of their own) of `prompt` tokens, KEPT of them kept, head by head;
    fewest..sharing sequences continue each; rows: own rows of a head before the step, at most."""
    return {"name": name, "do": "decode_shared", "q_heads": geometry[0], "kv_heads": geometry[1], "dim": geometry[2],
            "prompts": prompts, "prompt": prompt, "fewest": fewest or sharing, "sharing": sharing, "rows": rows,
            "capacity": capacity, "weights": weights, "sizes_seed": sizes_seed}


def _evict(name, geometry, seqs, rows, budget, recent, capacity, ragged=False, sizes_seed=0):
    """rows: of a head (ragged: from a quarter of that), budget: what a head keeps (ragged: up to half more)."""
    return {"name": name, "do": "evict_accumulated", "q_heads": geometry[0], "kv_heads": geometry[1], "dim": geometry[2],
            "seqs": seqs, "rows": rows, "budget": budget, "recent": recent, "capacity": capacity, "ragged": ragged,
            "sizes_seed": sizes_seed}


def listed():
    return [
        # one layer of a short prompt, everything computed here: the smallest call, where launches count
        _accumulate("accumulate_1x700", (28, 4, 128), 1, 700),
        # one layer of a long prompt at once
        _accumulate("accumulate_1x8192", (28, 4, 128), 1, 8192),
        # a chunk of a chunked prefill against the cache so far, in a padded slab, the prefill's log-sum-exp at hand
        _accumulate("accumulate_chunk_2x20000", (32, 4, 128), 2, 20000, queries=1000, layout="slab", lse=True),
        # a ragged batch of wide heads, keys as a projection leaves them
        _accumulate("accumulate_6xragged_d256", (8, 2, 256), 6, 500, 6000, layout="token", sizes_seed=3),
        # four samples of a short prompt, their first tokens: the smallest step
        _step("step_4_of_2048", (28, 4, 128), 1, 2048, 4, 20, 256),
        # 32 samples of long audio, some hundred tokens in
        _step("step_32_of_32768", (28, 4, 128), 1, 32768, 32, 300, 512),
        # a serving batch: eight recordings, up to 24 sequences each, wide heads, no totals kept
        _step("step_8xragged_d256", (8, 2, 256), 8, 12000, 24, 700, 1024, fewest=1, weights=False, sizes_seed=5),
        # sequences that share nothing, each at the budget of its evicting cache
        _step("step_48_own_4096", (28, 4, 128), 0, 0, 48, 4095, 4224),
        # one step's eviction: every head lost one row's room to the new token
        _evict("evict_one_of_1025", (28, 4, 128), 64, 1025, 1024, 128, 1088),
        # the prompt was long and the cache is halved at once, budgets by head
        _evict("evict_half_of_8192", (32, 4, 128), 16, 8192, 4096, 256, 8192, ragged=True, sizes_seed=7),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    geometry = rng.choice(GEOMETRIES)
    q_heads, kv_heads, dim = geometry
    do = rng.choice(["accumulate", "decode_shared", "evict_accumulated"])
    if do == "accumulate":
        length = _spread(rng, 60, 20000)
        queries = rng.choice([0, 0, _spread(rng, 1, 2000)])
        # the weights of all queries: a third of the largest listed case at most
        most = 1.2e9
        if not queries and length * length * q_heads > most:
            queries = max(1, int(most / (length * q_heads)))
        queries = min(queries, length)
        items = max(1, min(_spread(rng, 1, 8), int(most / (length * (queries or length) * q_heads))))
        shortest = max(1, queries, length // rng.choice([1, 3, 10]))
        case = _accumulate("", geometry, items, min(shortest, length), length, queries,
                           rng.choice(["head", "token", "slab"]), rng.random() < 0.4, rng.randrange(1 << 20))
    elif do == "decode_shared":
        prompts = rng.choice([0, 1, 1, _spread(rng, 2, 8)])
        sharing = _spread(rng, 1, 48 if prompts < 2 else 24)
        prompt = _spread(rng, 300, 32768 if prompts < 2 else 12000) if prompts else 0
        rows = _spread(rng, 1, max(2, min(4000, int(1e8 / (max(1, prompts) * sharing * kv_heads * dim)))))
        case = _step("", geometry, prompts, prompt, sharing, rows, rows + rng.choice([1, 37, 256]),
                     rng.choice([1, sharing]) if prompts else sharing, rng.random() < 0.6, rng.randrange(1 << 20))
    else:
        rows = _spread(rng, 20, 9000)
        seqs = max(1, min(_spread(rng, 1, 64), int(6e7 / (rows * kv_heads * dim))))
        budget = max(1, rows - _spread(rng, 1, max(2, rows // 2)))
        case = _evict("", geometry, seqs, rows, budget, min(budget, rng.choice([1, 16, 128])),
                      rows + rng.choice([0, 5, 64]), rng.random() < 0.5, rng.randrange(1 << 20))
    del case["name"]
    return case


# ---- sizes ---------------------------------------------------------------------------------------------------------

def _lengths(case):
    r = random.Random(case["sizes_seed"])
    lo, hi = case["shortest"], case["longest"]
    lens = [_spread(r, lo, hi) if lo < hi else hi for _ in range(case["items"])]
    lens[0] = hi
    return lens, [min(case["queries"] or L, L) for L in lens]


def _step_sizes(case):
    """Rows that each head of each prompt kept, and the sequences that continue each prompt."""
    r = random.Random(case["sizes_seed"])
    if not case["prompts"]:
        return [], [case["sharing"]]
    budgets = []
    for _ in range(case["prompts"]):
        tokens = case["prompt"] if case["prompts"] == 1 else _spread(r, max(1, case["prompt"] // 8), case["prompt"])
        keep = max(1, int(tokens * KEPT))
        share = [r.uniform(0.4, 1.6) for _ in range(case["kv_heads"])]
        budgets += [max(1, min(tokens, int(keep * case["kv_heads"] * s / sum(share)))) for s in share]
    sharing = [_spread(r, case["fewest"], case["sharing"]) if case["fewest"] < case["sharing"] else case["sharing"]
               for _ in range(case["prompts"])]
    sharing[0] = case["sharing"]
    return budgets, sharing


def _evict_sizes(case):
    r = random.Random(case["sizes_seed"])
    heads = case["seqs"] * case["kv_heads"]
    if not case["ragged"]:
        return [case["rows"]] * heads, [case["budget"]] * heads
    rows = [r.randint(max(1, case["rows"] // 4), case["rows"]) for _ in range(heads)]
    return rows, [r.randint(case["budget"], case["budget"] + case["budget"] // 2) for _ in range(heads)]


def work(case):
    H, G, d = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"]
    if case["do"] == "accumulate":
        lens, queries = _lengths(case)
        pairs = sum(Q * (L - Q) + Q * (Q + 1) / 2 for L, Q in zip(lens, queries))
        values = sum(queries) * case["q_heads"] * (d * 2 + (4 if case["lse"] else 0)) + sum(lens) * H * (d * 2 + 8)
        # one product of queries and keys with the log-sum-exp at hand, two without
        return {"bytes": values, "flops": 2 * case["q_heads"] * d * pairs * (1 if case["lse"] else 2)}
    if case["do"] == "decode_shared":
        budgets, sharing = _step_sizes(case)
        seqs, rows = sum(sharing), case["rows"] + 1
        shared = sum(b * sharing[g // H] for g, b in enumerate(budgets))       # (row, sequence) pairs
        totals = seqs * H * rows * 8 if case["weights"] else 0
        return {"bytes": (sum(budgets) + seqs * H * (rows + 1)) * d * 4 + seqs * case["q_heads"] * d * 4 + totals,
                "flops": 4 * G * d * (shared + seqs * H * rows)}
    rows, budgets = _evict_sizes(case)
    gone = sum(max(0, n - b) for n, b in zip(rows, budgets))
    # the totals and positions of all rows; a row that moves is read and written (about the kept share of the last ones)
    moved = sum(max(0, n - b) * b / n for n, b in zip(rows, budgets))
    return {"bytes": sum(rows) * 8 + moved * d * 8 + gone * 4, "flops": sum(rows)}


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


def prepare(case, seed):
    H, Hq, d = case["kv_heads"], case["q_heads"], case["dim"]
    s = {"case": case}
    if case["do"] == "accumulate":
        lens, queries = _lengths(case)
        s |= {"lens": lens, "queries": queries, "cu": _cu(lens), "cu_q": _cu(queries), "longest": max(lens)}
        tokens = case["items"] * max(lens) if case["layout"] == "slab" else sum(lens)
        s["k"] = _rows((tokens * H, d), _gen(seed, 0), keys=True)
        s["q"] = _rows((sum(queries) * Hq, d), _gen(seed, 1)) * 1.5
        # what earlier chunks gave
        s["before"] = torch.rand(tokens * H, generator=_gen(seed, 2), device="cuda") * (3 if case["queries"] else 0)
        s["totals"] = s["before"].clone()
        if case["lse"]:      # of the same rows: what a prefill's attention returns
            s["lse"] = torch.cat([_lse_of(s, i) for i in range(len(queries))])
        return s
    if case["do"] == "decode_shared":
        budgets, sharing = _step_sizes(case)
        seqs, C = sum(sharing), case["capacity"]
        s |= {"budgets": budgets, "sharing": sharing, "seqs": seqs, "cu_seqs": _cu(sharing)}
        s["q"] = _rows((seqs, Hq, d), _gen(seed, 0)) * 1.5
        if budgets:
            s["cu_budgets"], s["k_prompt"] = _cu(budgets), _rows((sum(budgets), d), _gen(seed, 1), keys=True)
            s["v_prompt"] = _rows((sum(budgets), d), _gen(seed, 2))
        s["k_own"], s["v_own"] = _rows((seqs, H, C, d), _gen(seed, 3), keys=True), _rows((seqs, H, C, d), _gen(seed, 4))
        s["k_new"], s["v_new"] = _rows((seqs, H, d), _gen(seed, 5), keys=True), _rows((seqs, H, d), _gen(seed, 6))
        # lengths, positions and totals lie in one buffer, so that one copy takes a pass back to where it began
        n = seqs * H
        live = torch.zeros(n * (1 + 2 * C), dtype=torch.int32, device="cuda")
        lengths = torch.full((seqs, 1), case["rows"], dtype=torch.int32, device="cuda").expand(seqs, H).clone()
        if case["prompts"] != 1:       # sequences that began at different times
            lengths = (torch.rand((seqs, 1), generator=_gen(seed, 7), device="cuda") * case["rows"]).int().expand(seqs, H).clone()
            lengths[0] = case["rows"]
        live[:n] = lengths.reshape(-1)
        live[n:n * (1 + C)] = torch.arange(C, dtype=torch.int32, device="cuda").repeat(n)
        live[n * (1 + C):].view(torch.float32).copy_(torch.rand(n * C, generator=_gen(seed, 8), device="cuda").square() * 4)
        s["pos"] = (10_000 + lengths[:, 0]).contiguous()
        s["live"], s["begin"] = live, live.clone()
        return s
    rows, budgets = _evict_sizes(case)
    n, C = case["seqs"] * H, case["capacity"]
    s |= {"rows": rows, "budget_list": budgets, "budgets": torch.tensor(budgets, dtype=torch.int32, device="cuda")}
    s["k_own"], s["v_own"] = _rows((case["seqs"], H, C, d), _gen(seed, 0)), _rows((case["seqs"], H, C, d), _gen(seed, 1))
    live = torch.zeros(n * (1 + 2 * C), dtype=torch.int32, device="cuda")
    live[:n] = torch.tensor(rows, dtype=torch.int32, device="cuda")
    # slots have been reused: their order is not that of time
    live[n:n * (1 + C)] = torch.rand((n, C), generator=_gen(seed, 2), device="cuda").argsort(dim=1).int().reshape(-1)
    totals = torch.exp(2 * torch.randn((n, C), generator=_gen(seed, 3), device="cuda"))
    totals[torch.rand((n, C), generator=_gen(seed, 4), device="cuda") < 0.02] = 0        # never looked at: equal totals
    live[n * (1 + C):].view(torch.float32).copy_(totals.reshape(-1))
    s["live"], s["begin"] = live, live.clone()
    return s


def _parts(s):
    """Lengths, positions and totals in the buffer that holds all three."""
    case, live = s["case"], s["live"]
    C = case["capacity"]
    n = live.numel() // (1 + 2 * C)
    return live[:n], live[n:n * (1 + C)].view(n, C), live[n * (1 + C):].view(torch.float32).view(n, C)


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _where(s):
    """Rows of K and of Q in their buffers for every (item, head, token) and (item, query head, query), lengths filled up,
    and which of them are there."""
    case, H, Hq = s["case"], s["case"]["kv_heads"], s["case"]["q_heads"]
    dev = s["k"].device
    L, Q = torch.tensor(s["lens"], device=dev)[:, None, None], torch.tensor(s["queries"], device=dev)[:, None, None]
    at, at_q = s["cu"].long()[:-1, None, None], s["cu_q"].long()[:-1, None, None]
    h, hq = torch.arange(H, device=dev)[None, :, None], torch.arange(Hq, device=dev)[None, :, None]
    j, i = torch.arange(max(s["lens"]), device=dev), torch.arange(max(s["queries"]), device=dev)
    if case["layout"] == "slab":
        row = (torch.arange(case["items"], device=dev)[:, None, None] * H + h) * s["longest"] + j
        row_w = row
    else:
        row = (at + j) * H + h if case["layout"] == "token" else at * H + h * L + j
        row_w = at * H + h * L + j
    row_q = (at_q + i) * Hq + hq if case["layout"] == "token" else at_q * Hq + hq * Q + i
    return row, row_w, row_q, (j < L).expand_as(row), (i < Q).expand_as(row_q)


def _logits(s, item=None):
    """[items, H, G, queries, tokens] in 32 bits, -inf where a query does not see a token or either is not there."""
    case = s["case"]
    H, G, d = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"]
    row, row_w, row_q, there, there_q = _where(s)
    pick = slice(None) if item is None else slice(item, item + 1)
    row, row_q, there, there_q = row[pick], row_q[pick], there[pick], there_q[pick]
    n, _, T = row.shape
    Q = row_q.shape[2]
    k = s["k"].float()[torch.where(there, row, 0)].view(n * H, T, d)
    q = s["q"].float()[torch.where(there_q, row_q, 0)].view(n * H, G * Q, d)
    z = torch.bmm(q, k.transpose(1, 2).contiguous()).view(n, H, G, Q, T).mul_(1 / math.sqrt(d))
    lens = torch.tensor(s["lens"][pick], device=z.device).view(n, 1, 1, 1, 1)
    queries = torch.tensor(s["queries"][pick], device=z.device).view(n, 1, 1, 1, 1)
    i, j = torch.arange(Q, device=z.device).view(-1, 1), torch.arange(T, device=z.device)
    return z.masked_fill_((j > lens - queries + i) | (j >= lens) | (i >= queries), -math.inf)


def _lse_of(s, item):
    """Log-sum-exp of an item's query rows, in the order of q without the head's channels."""
    z = _logits(s, item)[0]                                                    # [H, G, queries of the longest, T]
    z = z[:, :, :s["queries"][item]].double()
    m = z.amax(-1, keepdim=True)
    lse = (m.squeeze(-1) + (z - m).exp_().sum(-1).log()).float().flatten(0, 1)  # [Hq, Q]
    return lse.reshape(-1)


def _lse_rows(s):
    """The given log-sum-exp as [items, H, G, queries, 1]: fp32 [Hq][Q] of item after item."""
    case = s["case"]
    dev, Hq = s["lse"].device, case["q_heads"]
    i = torch.arange(max(s["queries"]), device=dev)
    Q, at = torch.tensor(s["queries"], device=dev)[:, None, None], s["cu_q"].long()[:-1, None, None]
    row = at * Hq + torch.arange(Hq, device=dev)[None, :, None] * Q + i
    there = (i < Q).expand_as(row)
    lse = torch.where(there, s["lse"][torch.where(there, row, 0)], math.inf)
    return lse.view(len(s["queries"]), case["kv_heads"], -1, len(i), 1)


def _plain_accumulate(s):
    z = _logits(s)
    if "lse" in s:
        p = z.sub_(_lse_rows(s)).exp_()
    else:
        m = z.amax(-1, keepdim=True)
        p = z.sub_(torch.where(m > -math.inf, m, 0.0)).exp_()
        p.div_(p.sum(-1, keepdim=True).clamp_min_(1e-38))
    got = p.sum(dim=(2, 3))                                                    # [items, H, T]
    _, row_w, _, there, _ = _where(s)
    s["totals"].copy_(s["before"])
    s["totals"][row_w[there]] += got[there]
    return s["totals"]


def _plain_step(s):
    case = s["case"]
    H, Hq, d = case["kv_heads"], case["q_heads"], case["dim"]
    G, n, dev = Hq // H, s["seqs"], s["q"].device
    s["live"].copy_(s["begin"])
    lengths, positions, totals = _parts(s)
    # the new row
    head = torch.arange(n * H, device=dev)
    slot = lengths.long()
    s["k_own"].view(n * H, -1, d)[head, slot] = s["k_new"].view(-1, d)
    s["v_own"].view(n * H, -1, d)[head, slot] = s["v_new"].view(-1, d)
    positions[head, slot] = s["pos"].repeat_interleave(H)
    if case["weights"]:
        totals[head, slot] = 0
    lengths += 1
    rows = case["rows"] + 1
    q = s["q"].float().view(n * H, G, d)
    k, v = s["k_own"].view(n * H, -1, d)[:, :rows].float(), s["v_own"].view(n * H, -1, d)[:, :rows].float()
    there = torch.arange(rows, device=dev) < lengths[:, None]
    z = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1 / math.sqrt(d)).masked_fill_(~there[:, None], -math.inf)
    m = z.amax(-1)
    if s["budgets"]:
        at = s["cu_budgets"].long()
        most, items = max(s["budgets"]), case["prompts"]
        j = torch.arange(most, device=dev)
        kept = j < (at[1:] - at[:-1])[:, None]                                 # [items * H, most]
        row = torch.where(kept, at[:-1, None] + j, 0)
        # sequences of an item side by side: [items, most sequences]
        first, S = s["cu_seqs"].long(), max(s["sharing"])
        seq = first[:-1, None] + torch.arange(S, device=dev)
        mine = seq < first[1:, None]
        qi = s["q"].float()[torch.where(mine, seq, 0)].view(items, S, H, G, d).transpose(1, 2).reshape(items * H, S * G, d)
        zi = torch.bmm(qi, s["k_prompt"].float()[row].transpose(1, 2).contiguous()).mul_(1 / math.sqrt(d)).masked_fill_(~kept[:, None], -math.inf)
        item = torch.repeat_interleave(torch.arange(items, device=dev), torch.tensor(s["sharing"], device=dev))
        nth = torch.arange(n, device=dev) - first[item]

        def by_sequence(x):            # [items * H, S * G, ...] -> [n * H, G, ...]
            return x.view(items, H, S, G, *x.shape[2:]).transpose(1, 2)[item, nth].reshape(n * H, G, *x.shape[2:])
        m_all = torch.maximum(m, by_sequence(zi.amax(-1)))
        spread = torch.zeros((items, S, H, G), device=dev)
        spread[item, nth] = m_all.view(n, H, G)
        pi = zi.sub_(spread.transpose(1, 2).reshape(items * H, S * G, 1)).exp_()
        den, num = by_sequence(pi.sum(-1)), by_sequence(torch.bmm(pi, s["v_prompt"].float()[row].masked_fill_(~kept[:, :, None], 0)))
        m = m_all
    p = z.sub_(m[..., None]).exp_()
    all_den, all_num = p.sum(-1), torch.bmm(p, v.masked_fill_(~there[:, :, None], 0))
    if s["budgets"]:
        all_den, all_num = all_den + den, all_num + num
    out = (all_num / all_den[..., None]).view(n, Hq, d).to(torch.bfloat16)
    if case["weights"]:
        totals[:, :rows] += (p / all_den[..., None]).sum(1)
    return out, s["k_own"], s["v_own"], lengths, positions, totals


def _plain_evict(s):
    case, d = s["case"], s["case"]["dim"]
    s["live"].copy_(s["begin"])
    lengths, positions, totals = _parts(s)
    n, C = positions.shape
    slot = torch.arange(C, device=positions.device).expand(n, C)
    there, b = slot < lengths[:, None], torch.minimum(s["budgets"], lengths)[:, None]
    newest = positions.masked_fill(~there, -1).amax(1, keepdim=True)
    worth = totals.masked_fill(there & (positions > newest - case["recent"]), math.inf).masked_fill(~there, -math.inf)
    order = worth.sort(dim=1, descending=True, stable=True).indices            # equal ones: the lower slot first
    rank = torch.empty_like(order).scatter_(1, order, slot)
    kept = (rank < b) & there
    hole, mover = (slot < b) & ~kept, (slot >= b) & kept
    nth = hole.cumsum(1) - 1
    movers = (~mover).to(torch.int8).sort(dim=1, stable=True).indices          # their slots, ascending
    src = torch.where(hole, movers.gather(1, nth.clamp_min(0)), slot)
    most = max(s["budget_list"])
    head = torch.arange(n, device=slot.device)[:, None]
    for x in (s["k_own"].view(n, C, d), s["v_own"].view(n, C, d), positions, totals):
        x[:, :most] = x[head, src[:, :most]]
    lengths.copy_(b[:, 0])
    return s["k_own"], s["v_own"], lengths, positions, totals


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    do = state["case"]["do"]
    if own:
        return {"accumulate": _own_accumulate, "decode_shared": _own_step, "evict_accumulated": _own_evict}[do](state)
    return {"accumulate": _plain_accumulate, "decode_shared": _plain_step, "evict_accumulated": _plain_evict}[do](state)


def _params(A, case, **more):
    return A.Params(case["q_heads"], case["kv_heads"], case["dim"], 0, **more)


def _own_accumulate(s):
    import paper_2604_06694_amd as A
    case = s["case"]
    if "p" not in s:          # a program lays these out once
        d, T = case["dim"], s["longest"]
        slab = case["layout"] == "slab"
        s["p"] = (_params(A, case, kv_stride_item=case["kv_heads"] * T * d, kv_stride_head=T * d, kv_stride_tok=d) if slab else
                  _params(A, case, kv_layout=A.LAYOUT_TOKEN_MAJOR if case["layout"] == "token" else A.LAYOUT_HEAD_MAJOR))
        s["pitch"] = T if slab else 0
        s["ws"] = torch.empty(max(256, A.accumulate_workspace_bytes(s["p"], s["lens"], s["queries"])), dtype=torch.uint8, device="cuda")
    s["totals"].copy_(s["before"])
    return A.accumulate(s["p"], s["q"], s["k"], s["lens"], s["queries"], weights=s["totals"], pitch=s["pitch"],
                        lse=s.get("lse"), cu_seqlens=s["cu"], cu_queries=s["cu_q"], workspace=s["ws"])


def _slots(A, s):
    lengths, positions, totals = _parts(s)
    return A.Slots(s["k_own"], s["v_own"], lengths, s["case"]["capacity"], positions=positions,
                   weights=totals if s["case"].get("weights", True) else None)


def _own_step(s):
    import paper_2604_06694_amd as A
    case = s["case"]
    if "p" not in s:
        s["p"], s["slots"] = _params(A, case), _slots(A, s)
        s["out"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
        s["ws"] = torch.empty(max(256, A.decode_shared_workspace_bytes(
            s["p"], case["prompts"], sum(s["budgets"]), s["seqs"], max(s["sharing"]), case["rows"] + 1)), dtype=torch.uint8, device="cuda")
    s["live"].copy_(s["begin"])
    A.decode_shared(s["p"], s["q"], s.get("k_prompt"), s.get("v_prompt"), s.get("cu_budgets"), sum(s["budgets"]),
                    s["cu_seqs"] if s["budgets"] else None, max(s["sharing"]), slots=s["slots"], max_own=case["rows"] + 1,
                    k_new=s["k_new"], v_new=s["v_new"], pos_new=s["pos"], out=s["out"], workspace=s["ws"])
    lengths, positions, totals = _parts(s)
    return s["out"], s["k_own"], s["v_own"], lengths, positions, totals


def _own_evict(s):
    import paper_2604_06694_amd as A
    case = s["case"]
    if "p" not in s:
        s["p"], s["slots"] = _params(A, case), _slots(A, s)
        s["ws"] = torch.empty(max(256, A.evict_accumulated_workspace_bytes(s["p"], case["seqs"], case["rows"], case["budget"])),
                              dtype=torch.uint8, device="cuda")
    s["live"].copy_(s["begin"])
    A.evict_accumulated(s["p"], s["slots"], case["seqs"], case["budget"], case["recent"], case["rows"],
                        budgets=s["budgets"] if case["ragged"] else None, workspace=s["ws"])
    lengths, positions, totals = _parts(s)
    return s["k_own"], s["v_own"], lengths, positions, totals


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    H, Hq, d = case["kv_heads"], case["q_heads"], case["dim"]
    G, scale = Hq // H, 1 / math.sqrt(case["dim"])
    if case["do"] == "accumulate":
        lens, queries, layout = s["lens"], s["queries"], case["layout"]
        totals = s["before"].double()
        at = at_q = 0
        for i, (L, Q) in enumerate(zip(lens, queries)):
            block, q = s["k"], s["q"][at_q * Hq:(at_q + Q) * Hq].double()
            if layout == "slab":
                keys = block.view(len(lens), H, s["longest"], d)[i, :, :L].double()
            elif layout == "token":
                keys = block[at * H:(at + L) * H].view(L, H, d).transpose(0, 1).double()
            else:
                keys = block[at * H:(at + L) * H].view(H, L, d).double()
            q = q.view(Q, Hq, d).transpose(0, 1) if layout == "token" else q.view(Hq, Q, d)
            for h in range(Hq):
                got = torch.zeros(L, dtype=torch.float64, device="cuda")
                for r in range(0, Q, 2048):
                    rows = q[h, r:r + 2048]
                    z = rows @ keys[h // G].T.contiguous() * scale
                    last = L - Q + r + torch.arange(len(rows), device="cuda")
                    z[torch.arange(L, device="cuda") > last[:, None]] = -math.inf
                    if case["lse"]:
                        e = s["lse"][at_q * Hq + h * Q + r:at_q * Hq + h * Q + r + len(rows)].double()
                        got += (z - e[:, None]).exp().sum(0)
                    else:
                        got += torch.softmax(z, dim=1).sum(0)
                where = (i * H + h // G) * s["longest"] if layout == "slab" else at * H + h // G * L
                totals[where:where + L] += got
            at, at_q = at + L, at_q + Q
        return totals
    live = s["live"].cpu().numpy()
    C = case["capacity"]
    n = live.size // (1 + 2 * C)
    lengths, positions = live[:n].copy(), live[n:n * (1 + C)].reshape(n, C).copy()
    totals = live[n * (1 + C):].view(np.float32).reshape(n, C).astype(np.float64)
    if case["do"] == "decode_shared":
        k, v = s["k_own"], s["v_own"]
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        pos, item, used = s["pos"].cpu().numpy(), 0, 0
        starts = np.concatenate([[0], np.cumsum(s["budgets"])]).astype(int)
        for x in range(s["seqs"]):
            while s["budgets"] and used == s["sharing"][item]:
                item, used = item + 1, 0
            used += 1
            for h in range(H):
                g = x * H + h
                m = int(lengths[g])
                k[x, h, m], v[x, h, m] = s["k_new"][x, h], s["v_new"][x, h]
                positions[g, m], lengths[g] = pos[x], m + 1
                keys, values = [k[x, h, :m + 1]], [v[x, h, :m + 1]]
                if s["budgets"]:
                    a, b = starts[item * H + h], starts[item * H + h + 1]
                    keys, values = [s["k_prompt"][a:b]] + keys, [s["v_prompt"][a:b]] + values
                z = s["q"][x, h * G:(h + 1) * G].double() @ torch.cat(keys).double().T.contiguous() * scale
                p = torch.softmax(z, dim=1)
                out[x, h * G:(h + 1) * G] = p @ torch.cat(values).double()
                if case["weights"]:
                    totals[g, m] = 0
                    totals[g, :m + 1] += p[:, -(m + 1):].sum(0).cpu().numpy()
        return out, k, v, lengths, positions, totals
    k, v = s["k_own"].view(n, C, d), s["v_own"].view(n, C, d)
    for g in range(n):
        rows, b = s["rows"][g], s["budget_list"][g]
        if rows <= b:
            continue
        newest = positions[g, :rows].max()
        order = sorted(range(rows), key=lambda t: (0 if positions[g, t] > newest - case["recent"] else 1,
                                                   0 if positions[g, t] > newest - case["recent"] else -totals[g, t], t))
        keep = set(order[:b])
        holes = [t for t in range(b) if t not in keep]
        movers = [t for t in range(b, rows) if t in keep]
        if holes:
            to, at = torch.tensor(holes, device="cuda"), torch.tensor(movers, device="cuda")
            k[g, to], v[g, to] = k[g, at], v[g, at]
            positions[g, holes], totals[g, holes] = positions[g, movers], totals[g, movers]
        lengths[g] = b
    return k.view(s["k_own"].shape), v.view(s["v_own"].shape), lengths, positions, totals
