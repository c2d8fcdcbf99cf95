"""The operators on a paged cache whose speed is followed: their calls, and the same in plain torch.

  append  norms of queries and keys for each head (where gains are given), the rotation by position, keys and values
          to their slots of the cache, queries in the cache's type
  attend  attention of the new rows of a batch of sequences over their slots, with the logarithm of each row's sum
  weigh   the attention weight that every slot got from these rows, added to what it had before
  evict   of every sequence and head the slots with the most weight, next to each other in new pages

The cache is [page][layer][k|v][kv_head][token in its page][head_dim].  A batch is `starts` (where each sequence's rows
begin, and the end of the last), `lengths` (slots in use, the new rows' among them, which are the last ones) and `table`
(the pages of each sequence).  Row i of a sequence with r rows and length n has slot n - r + i and sees the slots up to it.

Head counts and widths are those of the repository's backbones and test shape, and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}
EPS = 1e-6
DECAY = 0.75
FIRST, RECENT = 4, 32   # slots at a sequence's start and end that are always kept
BASE, LOW, HIGH, ORIGINAL = 10000.0, 1.0, 4.0, 8192


def listed():
    step, glm = dict(nq=28, nkv=4, hd=128), dict(nq=32, nkv=2, hd=128)
    return [
        # one speaker, one step: fp32 sums of the q/k/v product (latency)
        dict(name="append_step_1", op="append", n=1, rows=1, ctx=1025, **step, dtype="bf16", src="fp32", page=64, rotary=128, interleaved=False, norm=False, factor=1.0),
        # a long prompt on the other backbone: half of the head turned, in neighbouring pairs, far positions, norms
        dict(name="append_glm_8191", op="append", n=1, rows=8191, ctx=8191, **glm, dtype="bf16", src="bf16", page=64, rotary=64, interleaved=True, norm=True, factor=8.0),
        # a ragged batch of short prompts, small heads, small pages, all in fp32
        dict(name="append_odd_fp32", op="append", n=5, rows=203, ctx=611, nq=6, nkv=3, hd=64, dtype="fp32", src="fp32", page=16, rotary=64, interleaved=False, norm=True, factor=1.0),
        # one speaker, one step, behind a prompt of 512 and a response of 1024
        dict(name="attend_step_1", op="attend", n=1, rows=1, ctx=1537, **step, dtype="bf16", page=64),
        # a batch of 32 speakers with long dialogues, one step
        dict(name="attend_step_32", op="attend", n=32, rows=1, ctx=8191, **glm, dtype="bf16", page=64),
        # the next turn of a dialogue: a chunk over a cache
        dict(name="attend_chunk_511", op="attend", n=1, rows=511, ctx=2047, **step, dtype="bf16", page=64),
        # a long prompt in one go: matrix instructions
        dict(name="attend_prompt_8191", op="attend", n=1, rows=8191, ctx=8191, **step, dtype="bf16", page=64),
        # ragged chunks in fp32, small heads, pages that end inside a tile
        dict(name="attend_odd_fp32", op="attend", n=3, rows=100, ctx=1001, nq=4, nkv=2, hd=64, dtype="fp32", page=16),
        # weights gathered at a step of a batch
        dict(name="weigh_step_32", op="weigh", n=32, rows=1, ctx=4095, **step, dtype="bf16", page=64),
        # weights gathered once, from the last rows of a long prompt
        dict(name="weigh_window_64", op="weigh", n=1, rows=64, ctx=8191, **glm, dtype="bf16", page=64),
        # one dialogue cut to half
        dict(name="evict_one_4097", op="evict", n=1, ctx=4097, keep=2048, **step, dtype="bf16", page=64),
        # a batch of long dialogues cut to a quarter
        dict(name="evict_batch_32", op="evict", n=32, ctx=8191, keep=2000, **glm, dtype="bf16", page=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "weigh", "evict"])
    nq, nkv, hd = rng.choice([(28, 4, 128), (32, 2, 128), (4, 2, 64), (6, 3, 64), (16, 16, 64), (8, 8, 128), (24, 1, 128)])
    case = dict(op=op, nq=nq, nkv=nkv, hd=hd, dtype=rng.choice(["bf16", "bf16", "fp32"]), page=rng.choice([16, 32, 64, 80, 128]))
    if op == "append":
        rows = _log_int(rng, 1, 8000)
        case.update(n=_log_int(rng, 1, max(1, min(64, 8000 // rows))), rows=rows, ctx=rows + _log_int(rng, 1, 2000), src=rng.choice(["fp32", "bf16"]),
                    rotary=rng.choice([hd, hd, hd // 2, 24]), interleaved=rng.random() < 0.5, norm=rng.random() < 0.5, factor=rng.choice([1.0, 8.0]))
    elif op == "evict":
        ctx = _log_int(rng, 80, 8191)
        case.update(n=_log_int(rng, 1, max(1, min(48, 32 * 8191 * 2 // (ctx * nkv)))), ctx=ctx, keep=rng.randint(FIRST + RECENT, ctx))
    else:
        kind = rng.random()
        rows = 1 if kind < 0.4 else _log_int(rng, 2, 64) if kind < 0.7 or op == "weigh" else _log_int(rng, 64, 5000)
        ctx = rows + _log_int(rng, 1, 8000 - rows)
        most = min(64, 32 * 8191 * 2 // (ctx * nkv), (8191 * 8191 * 28 // 8) // (rows * ctx * nq))
        case.update(n=_log_int(rng, 1, max(1, most)), rows=rows, ctx=ctx)
    return case


def _shape(case):
    """(rows, length) of each sequence: the first has the most of both, the others less"""
    n, rows, ctx = case["n"], case.get("rows", 1), case["ctx"]
    return [(max(1, rows - (i * 13) % (rows // 2 + 1)), max(rows, ctx - (i * 997) % (ctx // 2 + 1))) for i in range(n)]


# ---------------------------------------------------------------------------------- inputs

def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * std

    n, nq, nkv, hd, page = (case[x] for x in ("n", "nq", "nkv", "hd", "page"))
    dtype, shape = DTYPES[case["dtype"]], _shape(case)
    pages = -(-case["ctx"] // page)
    out = {"table": torch.randperm(n * pages, generator=gen, device="cuda").view(n, pages).int(),
           "lengths": torch.tensor([c for _, c in shape], dtype=torch.int32, device="cuda"),
           "starts": torch.tensor([sum(r for r, _ in shape[:i]) for i in range(n + 1)], dtype=torch.int32, device="cuda")}
    m = sum(r for r, _ in shape)
    spare = -(-case["keep"] // page) if case["op"] == "evict" else 0
    if case["op"] == "append":
        out["pool"] = torch.zeros(n * pages, 1, 2, nkv, page, hd, dtype=dtype, device="cuda")
        src = DTYPES[case["src"]]
        qkv = normal(m, (nq + 2 * nkv) * hd) * torch.exp(0.3 * normal(m, 1))   # one product's outputs, read where they lie
        out["qkv"] = qkv.to(src)
        out["gains"] = [1 + 0.1 * normal(hd) for _ in range(2)] if case["norm"] else [None, None]
        # positions: those of the slots, or where older slots have gone, far ones
        far = 100000 if case["factor"] > 1 else 0
        first = out["lengths"].long() - (out["starts"][1:] - out["starts"][:-1])
        seq = torch.repeat_interleave(torch.arange(n, device="cuda"), (out["starts"][1:] - out["starts"][:-1]).long())
        out["positions"] = (torch.arange(m, device="cuda") - out["starts"][seq] + first[seq] + far).int()
        return out
    # a few channels of keys and values stand off zero, as in trained models
    pool = normal(n * pages + n * spare, 1, 2, nkv, page, hd) + normal(2, nkv, 1, hd, std=0.3)
    out["pool"] = pool.to(dtype)
    if case["op"] == "evict":
        # few slots get most of the weight, many none at all
        w = torch.exp(2 * normal(n, nkv, pages * page)) * (torch.rand(n, nkv, pages * page, generator=gen, device="cuda") < 0.8)
        used = torch.arange(pages * page, device="cuda") < out["lengths"][:, None, None]
        out["weights"] = w.bfloat16().float() * used
        out["table_out"] = (n * pages + torch.randperm(n * spare, generator=gen, device="cuda")).view(n, spare).int()
        return out
    out["q"] = normal(m, nq, hd, std=1.5).to(dtype)
    if case["op"] == "weigh":
        out["before"] = torch.exp(2 * normal(n, nkv, pages * page))
        out["lse"] = _row_sums(out["q"], out, max(r for r, _ in shape))
    return out


def prepare(case, seed):
    v = _inputs(case, seed)
    op, nq, nkv, hd = case["op"], case["nq"], case["nkv"], case["hd"]
    state = dict(v, op=op, case=case, max_rows=max(r for r, _ in _shape(case)))
    dtype, n = DTYPES[case["dtype"]], case["n"]
    slots = v["table"].shape[1] * case["page"]
    if op == "append":
        m = v["qkv"].shape[0]
        q, k, x = v["qkv"].split([nq * hd, nkv * hd, nkv * hd], dim=1)
        state.update(q=q.unflatten(1, (nq, hd)), k=k.unflatten(1, (nkv, hd)), v=x.unflatten(1, (nkv, hd)))
        state["out"] = torch.empty(m, nq, hd, dtype=dtype, device="cuda")
        state["freqs"] = _frequencies(case)
    elif op == "attend":
        state["out"] = torch.empty_like(v["q"])
        state["lse"] = torch.empty(v["q"].shape[:2], dtype=torch.float32, device="cuda")
    elif op == "weigh":
        state["out"] = torch.zeros(n, nkv, slots, dtype=torch.float32, device="cuda")
    else:
        state["weights_out"] = torch.zeros(n, nkv, slots, dtype=torch.float32, device="cuda")
    if own:
        from paper_2603_09215_amd import cached
        state["cache"] = cached.PagedCache(v["pool"])
        state["batch"] = cached.CachedRows(v["starts"], v["lengths"], v["table"])
        if op == "append":
            state["rotation"] = cached.Rotation(case["rotary"], base=BASE, interleaved=case["interleaved"], factor=case["factor"], low=LOW, high=HIGH,
                                                original=ORIGINAL, device="cuda")
    return state


# ---------------------------------------------------------------------------------- one pass

def run(state):
    op = state["op"]
    if own:
        from paper_2603_09215_amd import cached
        cache, batch = state["cache"], state["batch"]
        if op == "append":
            q_gain, k_gain = state["gains"]
            q = cached.cached_append(state["q"], state["k"], state["v"], cache, batch, rotation=state["rotation"], q_gain=q_gain, k_gain=k_gain, eps=EPS,
                                     positions=state["positions"], out=state["out"])
            return {"q": q, "pool": state["pool"]}
        if op == "attend":
            return {"out": cached.cached_attend(state["q"], cache, batch, out=state["out"], lse=state["lse"]), "lse": state["lse"]}
        if op == "weigh":
            return {"weights": cached.cached_weigh(state["q"], state["lse"], cache, batch, before=state["before"], decay=DECAY, out=state["out"])}
        kept, lengths = cached.cached_evict(cache, batch, state["weights"], state["case"]["keep"], first=FIRST, recent=RECENT, table_out=state["table_out"],
                                            weights_out=state["weights_out"])
        return {"kept": kept, "lengths": lengths, "weights": state["weights_out"], "pool": state["pool"]}
    return {"append": _append, "attend": _attend, "weigh": _weigh, "evict": _evict}[op](state)


def _frequencies(case):
    """the angle per position of each pair, in 64 bits; those of long waves are divided by the factor"""
    r = case["rotary"]
    f = BASE ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    turns = ORIGINAL * f / (2 * math.pi)
    stay = torch.clamp((turns - LOW) / (HIGH - LOW), 0, 1)
    return f * (stay + (1 - stay) / case["factor"])


def _turned(x, gain, angle, case):
    """norm and rotation of [m][heads][hd] in fp32; the angles in 64 bits"""
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    r, half = case["rotary"], case["rotary"] // 2
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :half], x[..., half:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _places(state):
    """(page, token in its page) of each row"""
    starts, lengths, table, page = state["starts"].long(), state["lengths"].long(), state["table"].long(), state["case"]["page"]
    seq = torch.repeat_interleave(torch.arange(table.shape[0], device="cuda"), starts[1:] - starts[:-1])
    slot = torch.arange(seq.shape[0], device="cuda") - starts[seq + 1] + lengths[seq]
    return table[seq, slot // page], slot % page


def _append(state):
    case, pool = state["case"], state["pool"]
    angle = state["positions"].double().unsqueeze(1) * state["freqs"]
    state["out"].copy_(_turned(state["q"], state["gains"][0], angle, case))
    page, token = _places(state)
    pool[page, 0, 0, :, token] = _turned(state["k"], state["gains"][1], angle, case).to(pool.dtype)
    pool[page, 0, 1, :, token] = state["v"].to(pool.dtype)
    return {"q": state["out"], "pool": pool}


def _of_cache(pool, table, which):
    """[n][nkv][slots][hd] in fp32"""
    return pool[table.long(), 0, which].transpose(1, 2).flatten(2, 3).float()


def _scores(q, batch, max_rows):
    """(scores [n][nkv][group * max_rows][slots], -inf where a row does not see; the rows [n][max_rows] of q, which of them are)"""
    table, starts, lengths = batch["table"], batch["starts"].long(), batch["lengths"].long()
    n, (m, nq, hd), nkv = table.shape[0], q.shape, batch["pool"].shape[3]
    k = _of_cache(batch["pool"], table, 0)
    row = starts[:-1, None] + torch.arange(max_rows, device="cuda")
    live = row < starts[1:, None]
    x = q[row.clamp(max=m - 1)].float().view(n, max_rows, nkv, nq // nkv, hd).permute(0, 2, 3, 1, 4).reshape(n, nkv, -1, hd)
    s = torch.matmul(x, k.transpose(-1, -2).contiguous()) * hd ** -0.5
    last = lengths[:, None] + row - starts[1:, None]
    hidden = torch.arange(s.shape[-1], device="cuda") > torch.where(live, last, 0)[:, :, None]
    s.view(n, nkv, nq // nkv, max_rows, -1).masked_fill_(hidden[:, None, None], -math.inf)
    return s, row, live


def _to_rows(x, live, nq):
    """[n][nkv][group * max_rows][...] -> [m][nq][...]"""
    n, max_rows = live.shape
    x = x.unflatten(2, (-1, max_rows)).flatten(1, 2).transpose(1, 2)   # [n][max_rows][nq][...]
    return x[live]


def _row_sums(q, batch, max_rows):
    """the logarithm of each row's sum, as an earlier pass of attention has left it"""
    s, _, live = _scores(q, batch, max_rows)
    top = s.amax(-1)
    return _to_rows(top + torch.log(torch.exp(s - top.unsqueeze(-1)).sum(-1)), live, q.shape[1]).contiguous()


def _attend(state):
    s, _, live = _scores(state["q"], state, state["max_rows"])
    top = s.amax(-1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, _of_cache(state["pool"], state["table"], 1)) / total
    nq = state["q"].shape[1]
    state["out"].copy_(_to_rows(out, live, nq))
    state["lse"].copy_(_to_rows((top + torch.log(total)).squeeze(-1), live, nq))
    return {"out": state["out"], "lse": state["lse"]}


def _weigh(state):
    s, row, live = _scores(state["q"], state, state["max_rows"])
    n, nkv = s.shape[:2]
    lse = state["lse"][row.clamp(max=state["lse"].shape[0] - 1)]   # [n][max_rows][nq]
    lse = torch.where(live.unsqueeze(-1), lse, math.inf).transpose(1, 2).reshape(n, nkv, -1)
    used = torch.arange(s.shape[-1], device="cuda") < state["lengths"][:, None, None]
    total = DECAY * state["before"] + torch.exp(s - lse.unsqueeze(-1)).sum(2)
    state["out"].copy_(torch.where(used, total, state["out"]))
    return {"weights": state["out"]}


def _evict(state):
    case, pool, lengths = state["case"], state["pool"], state["lengths"].long()
    keep, page, w = case["keep"], case["page"], state["weights"]
    slot = torch.arange(w.shape[-1], device="cuda")
    n_kept = torch.clamp(lengths, max=keep)
    always = (slot < FIRST) | (slot >= lengths[:, None, None] - RECENT)
    key = torch.where(slot < lengths[:, None, None], torch.where(always, math.inf, w), -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    there = (torch.arange(order.shape[-1], device="cuda") < n_kept[:, None, None]).expand_as(order)
    kept = torch.sort(torch.where(there, order, w.shape[-1]), dim=-1).values
    at = torch.where(there, kept, 0)
    n, nkv = kept.shape[:2]
    head = torch.arange(nkv, device="cuda")[None, :, None]
    src = torch.gather(state["table"].long(), 1, (at // page).flatten(1)).view_as(at)
    out = torch.arange(at.shape[-1], device="cuda")
    dst = state["table_out"].long()[:, out // page][:, None].expand_as(at)
    to = dst[there], head.expand_as(at)[there], (out % page).expand_as(at)[there]
    pool[to[0], 0, 0, to[1], to[2]] = pool[src, 0, 0, head, at % page][there]
    pool[to[0], 0, 1, to[1], to[2]] = pool[src, 0, 1, head, at % page][there]
    moved = torch.nn.functional.pad(torch.where(there, torch.gather(w, 2, at), 0.0), (0, w.shape[-1] - at.shape[-1]))
    state["weights_out"].copy_(torch.where(slot < lengths[:, None, None], moved, state["weights_out"]))
    return {"kept": torch.where(there, kept, -1).int(), "lengths": n_kept.int(), "weights": state["weights_out"], "pool": pool}


# ---------------------------------------------------------------------------------- what a pass needs

def work(case):
    op, nq, nkv, hd, size = case["op"], case["nq"], case["nkv"], case["hd"], SIZE[case["dtype"]]
    shape = _shape(case)
    m = sum(r for r, _ in shape)
    slots = sum(c for _, c in shape)
    if op == "append":
        return {"bytes": m * (nq + 2 * nkv) * hd * (SIZE[case["src"]] + size), "flops": 6.0 * m * (nq + nkv) * hd}
    if op == "evict":
        kept = sum(min(c, case["keep"]) for _, c in shape)
        return {"bytes": 4 * nkv * kept * hd * size + nkv * (8 * slots + 4 * kept), "flops": 2.0 * nkv * slots}
    seen = sum(r * c - r * (r - 1) // 2 for r, c in shape)   # (row, slot) pairs
    rows = m * nq * hd * size
    if op == "attend":
        return {"bytes": 2 * slots * nkv * hd * size + 2 * rows + 4 * m * nq, "flops": 4.0 * seen * nq * hd}
    return {"bytes": slots * nkv * (hd * size + 8) + rows + 4 * m * nq, "flops": 2.0 * seen * nq * hd}


# ---------------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    v = _inputs(case, seed)
    op, nq, nkv, hd, page = (case[x] for x in ("op", "nq", "nkv", "hd", "page"))
    shape, group = _shape(case), case["nq"] // case["nkv"]
    ends = [sum(r for r, _ in shape[:i + 1]) for i in range(case["n"])]
    pool = v["pool"]

    def plane(i, which):
        """[nkv][length][hd] of a sequence"""
        own_pages = pool[v["table"][i].long(), 0, which].double()           # [pages][nkv][page][hd]
        return torch.cat(list(own_pages), 1)[:, :shape[i][1]]

    if op == "append":
        out, heads = pool.double(), v["qkv"].double().view(-1, nq + 2 * nkv, hd)
        pair = torch.arange(case["rotary"] // 2, dtype=torch.float64, device="cuda")
        freq = torch.exp(-2 * pair / case["rotary"] * math.log(BASE))
        part = ((ORIGINAL * freq / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        freq = part * freq + (1 - part) * freq / case["factor"]
        turn = torch.polar(torch.ones_like(freq)[None], v["positions"].double()[:, None] * freq)[:, None]   # complex [m][1][pairs]

        def turned(x, gain):
            if gain is not None:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / hd + EPS) * gain.double()
            r = case["rotary"]
            first = slice(0, r, 2) if case["interleaved"] else slice(0, r // 2)
            second = slice(1, r, 2) if case["interleaved"] else slice(r // 2, r)
            z = torch.complex(x[..., first], x[..., second]) * turn
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y

        q, k = turned(heads[:, :nq], v["gains"][0]), turned(heads[:, nq:nq + nkv], v["gains"][1])
        at = 0
        for i, (r, c) in enumerate(shape):
            slot = torch.arange(c - r, c, device="cuda")
            place = v["table"][i].long()[torch.div(slot, page, rounding_mode="floor")]
            out[place, 0, 0, :, slot % page] = k[at:at + r]
            out[place, 0, 1, :, slot % page] = heads[at:at + r, nq + nkv:]
            at += r
        return {"q": q, "pool": out}
    if op == "evict":
        out, weights = pool.double(), torch.zeros_like(v["weights"], dtype=torch.float64)
        for i, (_, c) in enumerate(shape):
            left = min(c, case["keep"])
            for h in range(nkv):
                w = v["weights"][i, h, :c].double().clone()
                w[:FIRST], w[max(0, c - RECENT):] = math.inf, math.inf
                # ranked by weight, then by slot
                rank = torch.sort(-w, stable=True).indices[:left]
                kept = torch.sort(rank).values
                weights[i, h, :left] = v["weights"][i, h, kept].double()
                to = torch.arange(left, device="cuda")
                for which in (0, 1):
                    out[v["table_out"][i].long()[to // page], 0, which, h, to % page] = plane(i, which)[h, kept]
        return {"kept": None, "lengths": None, "weights": weights, "pool": out}
    if op == "attend":
        m = ends[-1]
        result, sums = torch.empty(m, nq, hd, dtype=torch.float64, device="cuda"), torch.empty(m, nq, dtype=torch.float64, device="cuda")
    else:
        total = torch.zeros(v["before"].shape, dtype=torch.float64, device="cuda")
    for i, (r, c) in enumerate(shape):
        q = v["q"][ends[i] - r:ends[i]].double()
        keys, values = plane(i, 0), plane(i, 1)
        sees = torch.arange(c, device="cuda")[None] <= torch.arange(c - r, c, device="cuda")[:, None]
        for h in range(nq):
            s = (q[:, h] @ keys[h // group].t().contiguous()) / math.sqrt(hd)
            s = s.masked_fill(~sees, -math.inf)
            if op == "attend":
                sums[ends[i] - r:ends[i], h] = torch.logsumexp(s, 1)
                result[ends[i] - r:ends[i], h] = torch.softmax(s, 1) @ values[h // group]
            else:
                total[i, h // group, :c] += torch.exp(s - v["lse"][ends[i] - r:ends[i], h, None].double()).sum(0)
        if op == "weigh":
            total[i, :, :c] += DECAY * v["before"][i, :, :c].double()
    return {"out": result, "lse": sums} if op == "attend" else {"weights": total}
