"""Cases on which the operators of a serving step over a 4-bit cache are measured.

``op`` names the operator:

  "pages"   block tables and slot map of a step: pages behind a request's end go back to the free stack, missing ones come from it
  "append"  queries and keys rotated, keys and values appended to the paged cache as blocks of 32 4-bit elements
  "attend"  causal attention of the new tokens over the 4-bit cache
  "probs"   logits to probabilities: repeated tokens penalised, biases, grammar masks, temperature, softmax

Batches are ragged: request r has ``cached`` tokens in front of ``new`` ones.  Lengths come from the case alone
(``lengths_seed``), so that its work does not depend on the inputs' seed.

The 4-bit format (OCP MXFP4): 32 neighbouring elements of a head row share a scale 2^s and are 2^s times one of 0, 0.5, 1, 1.5,
2, 3, 4, 6 with a sign, two codes to a byte, the first in the lower half.  A page of one head is its rows' code bytes and behind
them its rows' scale bytes (s + 127).
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 32
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _cache(name, op, heads, head_dim, batch, cached, new, **more):
    case = {"name": name, "op": op, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "batch": batch,
            "cached_lo": cached[0], "cached_hi": cached[1], "new_lo": new[0], "new_hi": new[1], "misses": 0, "miss_lo": 0,
            "miss_hi": 0, "page": 16, "base": 1.0e6, "rotary": head_dim, "interleaved": 0, "lengths_seed": 1}
    case.update(more)
    return case


def _pages(name, batch, cached, new, **more):
    case = {"name": name, "op": "pages", "batch": batch, "cached_lo": cached[0], "cached_hi": cached[1], "new_lo": new[0],
            "new_hi": new[1], "misses": 0, "miss_lo": 0, "miss_hi": 0, "finished": 0, "refused": 0, "page": 16, "lengths_seed": 1}
    case.update(more)
    return case


def _probs(name, batch, vocab, drafts, history, **more):
    case = {"name": name, "op": "probs", "batch": batch, "vocab": vocab, "drafts_lo": drafts[0], "drafts_hi": drafts[1],
            "history_lo": history[0], "history_hi": history[1], "bf16": True, "penalties": True, "biases": 32, "masked": 0.5,
            "lengths_seed": 1}
    case.update(more)
    return case


def listed():
    return [
        # next token of 16 users: most steps of a service
        _pages("pages_users", 16, (1024, 4096), (1, 1)),
        # a step that mixes increments behind refused drafts, whole new prompts and users that have left
        _pages("pages_mixed", 64, (512, 8192), (1, 256), misses=24, miss_lo=1024, miss_hi=4096, finished=8, refused=15),
        # next token of 16 users: the launch alone
        _cache("append_users", "append", (28, 4), 128, 16, (1024, 4096), (1, 1)),
        # a step that mixes cache hits with whole new prompts
        _cache("append_mixed", "append", (32, 8), 128, 64, (512, 8192), (1, 256), misses=32, miss_lo=1024, miss_hi=4096),
        # one user's next token: latency
        _cache("attend_user", "attend", (32, 8), 128, 1, (2344, 2344), (1, 1)),
        # next token of 32 users with long contexts
        _cache("attend_decode", "attend", (28, 4), 128, 32, (2048, 8192), (1, 1)),
        # five drafted tokens of each of 16 users
        _cache("attend_drafts", "attend", (32, 8), 128, 16, (1024, 4096), (6, 6)),
        # increments of an editor session behind cached prefix and suffix
        _cache("attend_extend", "attend", (28, 4), 128, 32, (2048, 8192), (8, 64)),
        # whole new prompts
        _cache("attend_prompts", "attend", (32, 8), 128, 8, (0, 0), (1024, 4096)),
        # five drafted tokens of one user, a vocabulary of the service's size
        _probs("probs_user", 1, 32004, (5, 5), (2355, 2355)),
        # up to 15 drafted tokens of 64 users, a large vocabulary of odd size
        _probs("probs_users", 64, 128003, (1, 15), (512, 8192)),
    ]


#: what the largest listed case costs, as an estimate that weighs bytes and operations
_MOST = 0.8e-3
#: and the most numbers that its scores, or four times its keys, are where every request is as long as the longest
_NUMBERS = 4.5e9


def _estimate(case):
    w = work(case)
    return w["bytes"] / 4.0e12 + w["flops"] / 0.7e15


def _numbers(case):
    if case["op"] != "attend":
        return 0
    rows = _lengths(case)
    keys = len(rows) * max(c + n for c, n in rows)
    return keys * max(case["q_heads"] * max(n for _, n in rows), 4 * case["kv_heads"] * case["head_dim"])


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pages", "append", "attend", "attend", "attend", "probs"])
    seed = rng.randrange(1, 1 << 20)
    if op == "probs":
        lo, past = rng.randint(0, 15), _log(rng, 1, 8192)
        case = _probs("", _log(rng, 1, 64), _log(rng, 4000, 160000), (lo, rng.randint(lo, 15)),
                      (past, min(16384, int(past * rng.uniform(1.0, 4.0)))), bf16=rng.random() < 0.7, penalties=rng.random() < 0.8,
                      biases=rng.choice([0, 1, 32, 300]), masked=rng.choice([0.0, 0.5, 1.0]), lengths_seed=seed)
        del case["name"]
        while _estimate(case) > _MOST:
            case["batch"] = max(1, case["batch"] // 2)
        return case
    batch, lo = _log(rng, 1, 64), _log(rng, 64, 8192)
    cached = (lo, min(16384, int(lo * rng.uniform(1.0, 4.0))))
    more = {"page": rng.choice([16, 16, 16, 8, 32, 64, 256]), "lengths_seed": seed}
    n = _log(rng, 1, 512)
    new = rng.choice([(1, 1), (1, 16), (6, 6), (n, int(n * rng.uniform(1.0, 4.0)))])
    if op == "attend" and rng.random() < 0.3:
        cached, n = (0, 0), _log(rng, 64, 2048)
        new = (n, 2 * n)
    if op != "attend" and rng.random() < 0.4:
        m = _log(rng, 512, 3000)
        more.update(misses=rng.randint(1, batch), miss_lo=m, miss_hi=min(4096, int(m * rng.uniform(1.0, 2.0))))
    if op == "pages":
        more.update(finished=rng.randint(0, batch // 2), refused=rng.choice([0, 0, 15]))
        case = _pages("", batch, cached, new, **more)
    else:
        heads, head_dim = rng.choice([((32, 8), 128), ((28, 4), 128), ((32, 32), 128), ((4, 4), 64), ((32, 8), 64)])
        case = _cache("", op, heads, head_dim, batch, cached, new, base=rng.choice([1.0e4, 5.0e5, 1.0e6]),
                      rotary=rng.choice([head_dim, head_dim, head_dim // 2]), interleaved=rng.choice([0, 0, 1]), **more)
    del case["name"]
    while op != "pages" and (_estimate(case) > _MOST or _numbers(case) > _NUMBERS):
        case["batch"] = max(1, case["batch"] // 2)
        case["misses"] = min(case["misses"], case["batch"])
        if case["batch"] == 1:
            for key in ("cached_lo", "cached_hi", "new_lo", "new_hi", "miss_lo", "miss_hi"):
                case[key] = -(-case[key] * 3 // 4)
    return case


def _lengths(case):
    """[(cached, new)] of the requests (of "probs": (history, drafted tokens)), the same for every seed."""
    rng = random.Random(case["lengths_seed"])
    if case["op"] == "probs":
        return [(rng.randint(case["history_lo"], case["history_hi"]), rng.randint(case["drafts_lo"], case["drafts_hi"]))
                for _ in range(case["batch"])]
    rows = []
    for r in range(case["batch"]):
        if r < case["misses"]:
            rows.append((0, rng.randint(case["miss_lo"], case["miss_hi"])))
        else:
            rows.append((rng.randint(case["cached_lo"], case["cached_hi"]), rng.randint(case["new_lo"], case["new_hi"])))
    rng.shuffle(rows)
    return rows


def _page_lengths(case):
    """[(held, cached, new)]: the tokens that a request's pages have been taken for, those that stay and the new ones."""
    rng = random.Random(case["lengths_seed"] + 1)
    rows = [(0 if c == 0 else c + rng.randint(0, case["refused"]), c, n) for c, n in _lengths(case)]
    for r in rng.sample(range(len(rows)), case["finished"]):
        rows[r] = (max(rows[r][0], 1), 0, 0)
    return rows


def work(case):
    if case["op"] == "probs":
        rows = sum(n + 1 for _, n in _lengths(case))
        past = sum(h for h, _ in _lengths(case)) if case["penalties"] else 0
        size = 2 if case["bf16"] else 4
        return {"bytes": int(rows * case["vocab"] * (size + 4 + case["masked"] / 8) + past * 4), "flops": 0}
    if case["op"] == "pages":
        rows, page = _page_lengths(case), case["page"]
        moved = sum(abs(-(-(c + n) // page) - -(-h // page)) for h, c, n in rows)
        return {"bytes": sum(n for _, _, n in rows) * 8 + moved * 8 + len(rows) * 16, "flops": 0}
    rows = _lengths(case)
    new, hq, hkv, d = sum(n for _, n in rows), case["q_heads"], case["kv_heads"], case["head_dim"]
    row = d // 2 + d // BLOCK
    if case["op"] == "append":
        return {"bytes": new * (hq * d * 4 + 2 * hkv * (d * 4 + row)), "flops": 0}
    pairs, keys = sum(n * c + n * (n + 1) // 2 for c, n in rows), sum(c + n for c, n in rows)
    return {"bytes": keys * hkv * 2 * row + new * hq * d * 4, "flops": 4 * d * hq * pairs}


# --- inputs ------------------------------------------------------------------------------------------------------------


def _table(need, extra, seed):
    """(block table, pages that no row has, pages) with disjoint pages in an order drawn from the seed."""
    pages = sum(need) + extra
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(need), max(max(need), 1)), int(order[-1]), dtype=torch.int32)
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = order[at:at + k]
        at += k
    return table, order[at:], pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "pages":
        return _prepare_pages(case, seed)
    if case["op"] == "probs":
        return _prepare_probs(case, gen)
    rows = _lengths(case)
    state = {"case": case, "rows": rows}

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        return torch.randn(shape, dtype=dtype, device="cuda", generator=gen).mul_(scale)

    cached, new = [c for c, _ in rows], [n for _, n in rows]
    total, hq, hkv, page, d = sum(new), case["q_heads"], case["kv_heads"], case["page"], case["head_dim"]
    need = [-(-(c + n) // page) for c, n in rows]
    table, _, pages = _table(need, max(2, sum(need) // 8), seed)  # an eighth of the pages unused
    state["table"] = table.cuda()
    # request, place in it and position of every new token: what an engine's step has at hand
    state["req"] = torch.repeat_interleave(torch.arange(len(rows)), torch.tensor(new)).cuda()
    state["place"] = torch.cat([torch.arange(n) for n in new]).cuda()
    state["cached"] = torch.tensor(cached).cuda()
    state["pos"] = state["cached"][state["req"]] + state["place"]
    state["inv_freq"] = case["base"] ** (-2.0 * np.arange(case["rotary"] // 2) / case["rotary"])
    state["q"] = normal(total, hq, d)
    shape = (pages, hkv, page * (d // 2 + d // BLOCK))
    if case["op"] == "append":
        # keys have a few channels that are much larger than the rest
        state["k"], state["v"] = normal(total, hkv, d), normal(total, hkv, d)
        state["k"][:, :, ::29] *= 6.0
        for name in ("k_cache", "v_cache"):
            state[name] = torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=gen)
        state["q_out"], state["k_stored"], state["v_stored"] = (torch.empty_like(state[x]) for x in "qkv")
    else:
        state["out"] = torch.empty_like(state["q"])
        for name in ("k_cache", "v_cache"):
            state[name] = torch.empty(shape, dtype=torch.uint8, device="cuda")
            codes, scales = _parts(state[name], case)
            for lo in range(0, pages, 1024):
                part = normal(min(1024, pages - lo), hkv, page, d, dtype=torch.float32)
                codes[lo:lo + 1024], scales[lo:lo + 1024] = _quantise(part)
    if own:
        from paper_2505_21889_amd import binding as E
        state["batch"] = E.BatchDesc(cached, new, state["table"], hq, hkv, d, page, pages)
        if case["op"] == "attend":
            state["ws_bytes"] = E.efim_mx4_workspace_bytes(state["batch"])
            state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device="cuda")
    return state


def _prepare_pages(case, seed):
    rows, page = _page_lengths(case), case["page"]
    held, wanted = [-(-h // page) for h, _, _ in rows], [-(-(c + n) // page) for _, c, n in rows]
    table, free, pages = _table(held, sum(wanted) + 64, seed)  # what is asked for is there
    wide = max(max(held), max(wanted), 1)
    table = torch.nn.functional.pad(table, (0, wide - table.shape[1]), value=0)
    state = {"case": case, "rows": rows, "table": table.cuda(), "pages": pages}
    state["held"], state["cached"], state["new"] = (torch.tensor([row[i] for row in rows], dtype=torch.int32).cuda() for i in range(3))
    stack = torch.full((pages,), -1, dtype=torch.int32)
    stack[:len(free)] = free
    state["free"], state["count"] = stack.cuda(), torch.tensor([len(free)], dtype=torch.int32).cuda()
    state["count_out"] = torch.empty_like(state["count"])
    # a step's slot map has places for more tokens than it has, as a captured step's does
    state["slots"] = torch.empty(sum(n for _, _, n in rows) + 16, dtype=torch.int64, device="cuda")
    state["row_start"] = torch.empty(len(rows) + 1, dtype=torch.int32, device="cuda")
    state["status"] = torch.empty(1, dtype=torch.int32, device="cuda")
    if own:
        from paper_2505_21889_amd import binding as E
        state["ws_bytes"] = E.efim_block_tables_workspace_bytes(len(rows))
        state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device="cuda")
    return state


def _prepare_probs(case, gen):
    rows, vocab, rng = _lengths(case), case["vocab"], random.Random(case["lengths_seed"] + 1)
    drafts = [n for _, n in rows]
    total, batch = sum(drafts) + len(rows), len(rows)
    state = {"case": case, "rows": rows}
    logits = torch.randn(total, vocab, device="cuda", generator=gen).mul_(3.0)
    state["logits"] = logits.to(torch.bfloat16) if case["bf16"] else logits

    def tokens(*shape):  # some words are much more frequent than others
        return (torch.rand(shape, device="cuda", generator=gen) ** 3 * vocab).int().clamp_(max=vocab - 1)

    state["history"] = tokens(batch, max(h for h, _ in rows))
    state["drafts"] = tokens(sum(drafts))
    state["bias_tokens"] = tokens(batch, max(case["biases"], 1))
    state["bias_values"] = torch.randn(batch, max(case["biases"], 1), device="cuda", generator=gen).mul_(4.0)
    params = torch.zeros(batch, 8)
    whole = params.view(torch.int32)
    for r, (h, _) in enumerate(rows):
        params[r, 0] = rng.choice([0.0, 0.6, 0.8, 1.0])  # temperature
        params[r, 1] = rng.choice([1.0, 1.1, 1.3]) if case["penalties"] else 1.0
        params[r, 2], params[r, 3] = (rng.choice([0.0, 0.5]), rng.choice([0.0, 0.2])) if case["penalties"] else (0.0, 0.0)
        whole[r, 4] = rng.randint(h // 2, h)  # of the history, the prompt
        whole[r, 5] = h
        whole[r, 6] = rng.randint(0, case["biases"])
    state["params"] = params.cuda()
    masks = max(1, int(total * case["masked"]))
    words = (vocab + 31) // 32
    bits = torch.randint(-2 ** 31, 2 ** 31, (masks, words), device="cuda", generator=gen).int()
    bits[::2] &= torch.randint(-2 ** 31, 2 ** 31, (len(bits[::2]), words), device="cuda", generator=gen).int()
    state["masks"] = bits
    chosen = [i if i < masks and case["masked"] > 0 else -1 for i in range(total)]
    rng.shuffle(chosen)
    state["mask_rows"] = torch.tensor(chosen, dtype=torch.int32).cuda()
    state["req"] = torch.repeat_interleave(torch.arange(batch), torch.tensor(drafts) + 1).cuda()
    state["place"] = torch.cat([torch.arange(n + 1) for n in drafts]).cuda()
    state["first"] = torch.tensor([0] + drafts[:-1]).cumsum(0).cuda()  # first drafted token of each request
    state["probs"] = torch.empty(total, vocab, device="cuda")
    if own:
        from paper_2505_21889_amd import binding as E
        state["desc"] = E.LogitsDesc(drafts, vocab, state["logits"], vocab, state["params"], state["history"],
                                     state["history"].shape[1], state["drafts"], state["bias_tokens"], state["bias_values"],
                                     state["bias_tokens"].shape[1], state["masks"], words, masks, state["mask_rows"])
        state["ws_bytes"] = E.efim_logit_workspace_bytes(state["desc"])
        state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device="cuda")
    return state


# --- the operators -------------------------------------------------------------------------------------------------------


def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _own_pages(s):
    from paper_2505_21889_amd import binding as E
    E.efim_block_tables(len(s["rows"]), s["held"], s["cached"], s["new"], s["case"]["page"], s["table"], s["table"].shape[1], s["free"],
                        s["pages"], s["count"], s["count_out"], s["slots"], len(s["slots"]), s["row_start"], s["status"], s["ws"],
                        s["ws_bytes"])
    return {"table": s["table"], "free": s["free"], "count": s["count_out"], "slots": s["slots"], "row_start": s["row_start"],
            "status": s["status"]}


def _own_append(s):
    from paper_2505_21889_amd import binding as E
    E.efim_rope_append_mx4(s["batch"], s["q"], s["q_out"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_stored"], s["v_stored"],
                           s["inv_freq"], s["case"]["rotary"], s["case"]["interleaved"])
    return {"q": s["q_out"], "k": s["k_stored"], "v": s["v_stored"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_attend(s):
    from paper_2505_21889_amd import binding as E
    E.efim_extend_attention_mx4(s["batch"], s["q"], s["k_cache"], s["v_cache"], s["out"], 0.0, s["ws"], s["ws_bytes"])
    return s["out"]


def _own_probs(s):
    from paper_2505_21889_amd import binding as E
    E.efim_logit_probs(s["desc"], s["probs"], s["case"]["vocab"], s["ws"], s["ws_bytes"])
    return s["probs"]


_run_own = {"pages": _own_pages, "append": _own_append, "attend": _own_attend, "probs": _own_probs}


def _plain_pages(s):
    page, table, free, cached, new = s["case"]["page"], s["table"].long(), s["free"].long(), s["cached"].long(), s["new"].long()
    held, wanted = -(-s["held"].long() // page), -(-(cached + new) // page)
    column = torch.arange(table.shape[1], device="cuda")
    back = (column >= wanted[:, None]) & (column < held[:, None])
    more = (column >= held[:, None]) & (column < wanted[:, None])
    # the pages of the rows' ends go onto the stack, request by request
    at = torch.where(back, s["count"] + back.flatten().cumsum(0).view_as(back) - 1, len(free))
    stack = torch.cat([free, free[:1]]).scatter_(0, at.flatten(), table.flatten())
    count = s["count"] + back.sum() - more.sum()
    rank = more.flatten().cumsum(0).view_as(more)
    fits = count >= 0
    place = (s["count"] + back.sum() - rank).clamp_(0, len(free) - 1)
    table = torch.where(more & fits, stack[place], table)
    free = torch.where(fits, stack[:-1], free)
    start = torch.cat([new.new_zeros(1), new.cumsum(0)])
    t = torch.arange(len(s["slots"]), device="cuda")
    req = (torch.searchsorted(start, t, right=True) - 1).clamp_(max=len(new) - 1)
    pos = (cached[req] + t - start[req]).clamp_(max=table.shape[1] * page - 1)
    slots = torch.where((t < start[-1]) & fits, table[req, pos // page] * page + pos % page, -1)
    return {"table": table.int(), "free": free.int(), "count": torch.where(fits, count, s["count"]).int(), "slots": slots,
            "row_start": start.int(), "status": (-count).clamp_(min=0).int()}


def _parts(cache, case):
    """Codes [pages, heads, page, head_dim / 2] and scales [.., head_dim / 32] of a cache, as views of it."""
    page, d = case["page"], case["head_dim"]
    return (cache[..., :page * d // 2].unflatten(-1, (page, d // 2)), cache[..., page * d // 2:].unflatten(-1, (page, d // BLOCK)))


def _quantise(x):
    """Codes and scale bytes of float rows [.., head_dim]."""
    x = x.unflatten(-1, (-1, BLOCK))
    size = x.abs()
    most = size.amax(-1)
    part, power = torch.frexp(most)  # most = part 2^power, 0.5 <= part < 1
    power = torch.where(most > 0, power - 3 + (part > 0.875), -125).clamp_(-125, 125)
    size = torch.ldexp(size, -power[..., None])
    # the middle between two levels goes to the one with an even code
    code = (size > 0.25).byte() + (size >= 0.75) + (size > 1.25) + (size >= 1.75) + (size > 2.5) + (size >= 3.5) + (size > 5.0)
    code += 8 * torch.signbit(x)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (power + 127).byte()


def _values(codes, scales):
    """Float rows of codes and scale bytes."""
    levels = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device="cuda")
    x = levels[torch.stack([codes & 15, codes >> 4], -1).int()].flatten(-2)
    return torch.ldexp(x.unflatten(-1, (-1, BLOCK)), scales.int()[..., None] - 127).flatten(-2)


def _rotate(x, s):
    """Rows [T, heads, d] rotated at the tokens' positions, rounded to bf16."""
    # (in 64 bits: codes follow from values next to a border)
    angle = s["pos"].double()[:, None] * torch.from_numpy(s["inv_freq"]).cuda()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    half = cos.shape[-1]
    y = x.clone()
    if s["case"]["interleaved"]:
        a, b = x[..., 0:2 * half:2].double(), x[..., 1:2 * half:2].double()
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = _bf16(a * cos - b * sin), _bf16(b * cos + a * sin)
    else:
        a, b = x[..., :half].double(), x[..., half:2 * half].double()
        y[..., :half], y[..., half:2 * half] = _bf16(a * cos - b * sin), _bf16(b * cos + a * sin)
    return y


def _bf16(x):
    """Doubles rounded once to bf16 (through 32 bits a value next to a middle would be rounded twice)."""
    y = x.float()
    middle = (y.view(torch.int32) & 0xFFFF) == 0x8000
    away = torch.sign(x.abs() - y.double().abs()).int()
    return torch.where(middle, (y.view(torch.int32) + away).view(torch.float32), y).to(torch.bfloat16)


def _plain_append(s):
    page = s["case"]["page"]
    at, slot = s["table"][s["req"], s["pos"] // page].long(), s["pos"] % page
    out = {"q": _rotate(s["q"], s)}
    for name, rows in (("k", _rotate(s["k"], s)), ("v", s["v"])):
        codes, scales = _parts(s[name + "_cache"], s["case"])
        codes[at, :, slot], scales[at, :, slot] = new = _quantise(rows.float())
        out[name] = _values(*new).to(torch.bfloat16)
    return {**out, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attend(s):
    case, table = s["case"], s["table"].long()
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    keys, values = (_values(*(x[table] for x in _parts(s[name], case))).transpose(1, 2).flatten(2, 3).flatten(0, 1)
                    for name in ("k_cache", "v_cache"))  # [batch * kv heads, keys, d]
    new = max(n for _, n in s["rows"])
    q = torch.zeros(len(table), new, hq, d, device="cuda")
    q[s["req"], s["place"]] = s["q"].float()
    q = q.unflatten(2, (hkv, -1)).transpose(1, 2).reshape(len(keys), -1, d)
    scores = torch.bmm(q, keys.transpose(1, 2).contiguous()).mul_(d ** -0.5).view(len(table), hkv, new, -1, keys.shape[1])
    last = s["cached"][:, None] + torch.arange(new, device="cuda")  # of the keys that a row sees
    hidden = torch.arange(keys.shape[1], device="cuda") > last[..., None]
    scores.masked_fill_(hidden[:, None, :, None], -math.inf)
    scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    scores.div_(scores.sum(-1, keepdim=True))
    out = torch.bmm(scores.view(len(keys), -1, keys.shape[1]), values).view(len(table), hkv, new, -1, d)
    return out.transpose(1, 2).reshape(len(table), new, hq, d)[s["req"], s["place"]].to(torch.bfloat16)


def _plain_probs(s):
    vocab, history, req, place = s["case"]["vocab"], s["history"].long(), s["req"], s["place"]
    params, whole = s["params"], s["params"].view(torch.int32)
    z = s["logits"].float()
    heat, repeat, presence, frequency = (params[req, i][:, None] for i in range(4))
    # how often a token has been seen, and seen behind the prompt
    column = torch.arange(history.shape[1], device="cuda")
    past = column < whole[:, 5:6]
    made = past & (column >= whole[:, 4:5])
    seen = torch.zeros(len(history), vocab, dtype=torch.int32, device="cuda").scatter_add_(1, history, past.int())[req]
    often = torch.zeros(len(history), vocab, dtype=torch.int32, device="cuda").scatter_add_(1, history, made.int())[req]
    if len(s["drafts"]):  # a row has seen the drafted tokens in front of it
        j = torch.arange(int(max(n for _, n in s["rows"])), device="cuda")
        front = s["drafts"][(s["first"][req][:, None] + j).clamp_(max=len(s["drafts"]) - 1)].long()
        counts = (j < place[:, None]).int()
        seen.scatter_add_(1, front, counts)
        often.scatter_add_(1, front, counts)
    z = torch.where(seen > 0, torch.where(z > 0, z / repeat, z * repeat), z)
    z = torch.where(often > 0, z - frequency * often - presence, z)
    # of several biases of a token the last one counts
    number = torch.arange(1, s["bias_tokens"].shape[1] + 1, device="cuda")
    number = torch.where(number <= whole[:, 6:7], number, 0)
    index = torch.zeros(len(history), vocab, dtype=torch.int64, device="cuda")
    index.scatter_reduce_(1, s["bias_tokens"].long(), number, "amax")
    bias = torch.where(index > 0, s["bias_values"].gather(1, (index - 1).clamp_(min=0)), 0.0)
    z = z + bias[req]
    t = torch.arange(vocab, device="cuda")
    bits = s["masks"][s["mask_rows"].clamp(min=0).long()][:, t // 32] >> (t % 32)
    z = z.masked_fill(((bits & 1) == 0) & (s["mask_rows"] >= 0)[:, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp((z - top) / torch.where(heat > 0, heat, 1.0))
    p = p / p.sum(-1, keepdim=True)
    greedy = (t == (z == top).int().argmax(-1, keepdim=True)).float()
    return torch.where(top == -math.inf, 0.0, torch.where(heat > 0, p, greedy))


_run_plain = {"pages": _plain_pages, "append": _plain_append, "attend": _plain_attend, "probs": _plain_probs}


# --- the definitions in 64 bits ------------------------------------------------------------------------------------------


def exact(case, seed):
    return _exact[case["op"]](prepare(case, seed))


def _exact_pages(s):
    page, table, stack = s["case"]["page"], s["table"].cpu().clone(), s["free"].tolist()
    count, slots = int(s["count"][0]), []
    for r, (h, c, n) in enumerate(s["rows"]):
        for col in range(-(-(c + n) // page), -(-h // page)):
            stack[count] = int(table[r, col])
            count += 1
    for r, (h, c, n) in enumerate(s["rows"]):
        for col in range(-(-h // page), -(-(c + n) // page)):
            count -= 1
            table[r, col] = stack[count]
        slots += [int(table[r, p // page]) * page + p % page for p in range(c, c + n)]
    start = np.concatenate([[0], np.cumsum([n for _, _, n in s["rows"]])]).astype(np.int32)
    slots = np.array(slots + [-1] * (len(s["slots"]) - len(slots)), dtype=np.int64)
    return {"table": table, "free": torch.tensor(stack, dtype=torch.int32), "count": torch.tensor([count], dtype=torch.int32),
            "slots": torch.from_numpy(slots), "row_start": torch.from_numpy(start), "status": torch.zeros(1, dtype=torch.int32)}


def _exact_append(s):
    case = s["case"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["pos"].double()[:, None] * torch.from_numpy(s["inv_freq"]).cuda())[:, None]
    half = turn.shape[-1]

    def turned(x):
        """Rows in 64 bits, pairs taken as complex numbers and multiplied by exp(i angle)."""
        x = x.double()
        lead = x[..., :2 * half].unflatten(-1, (half, 2) if case["interleaved"] else (2, half))
        if not case["interleaved"]:
            lead = lead.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(lead.contiguous()) * turn)
        if not case["interleaved"]:
            z = z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), x[..., 2 * half:]], -1)

    def stored(x):
        """What stands for rows in 64 bits, rounded to bf16 first: the nearest of all fifteen levels of a block's scale."""
        x = _bf16(x).double().unflatten(-1, (-1, BLOCK))
        most = x.abs().amax(-1, keepdim=True)
        power = torch.ceil(torch.log2(most.clamp(min=2.0 ** -140) / 7.0)).clamp_(-125, 125)
        x = x / 2.0 ** power
        # half a step between neighbours: 0.5 up to 2, 1 up to 4, 2 above
        step = torch.where(x.abs() < 2, 0.5, torch.where(x.abs() < 4, 1.0, 2.0))
        return (torch.round(x / step) * step).clamp_(-6, 6).mul_(2.0 ** power).flatten(-2)

    # (the caches' bytes are compared between the kernels and the plain form, and k and v are what they stand for)
    return {"q": turned(s["q"]), "k": stored(turned(s["k"])), "v": stored(s["v"].double()), "k_cache": None, "v_cache": None}


def _exact_attend(s):
    case, at = s["case"], 0
    page, hkv, d = case["page"], case["kv_heads"], case["head_dim"]
    g = case["q_heads"] // hkv
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")

    def rows(name, r, keys, h):
        """Rows [keys, d] of a request's kv head in 64 bits, number by number: (-1)^sign 2^exponent (1 + mantissa / 2)."""
        where = torch.arange(keys, device="cuda")
        block = s[name][s["table"][r].long()[where.div(page, rounding_mode="floor")], h]
        slot = where.remainder(page)[:, None]
        element = torch.arange(d, device="cuda")
        nibble = block.gather(1, slot * (d // 2) + element // 2) >> (4 * (element % 2)).to(torch.uint8)
        sign, power, part = 1.0 - 2.0 * (nibble >> 3 & 1).double(), (nibble >> 1 & 3).double(), (nibble & 1).double()
        size = torch.where(power == 0, part / 2, (1 + part / 2) * 2.0 ** (power - 1))
        scale = block.gather(1, page * (d // 2) + slot * (d // BLOCK) + element // BLOCK).double()
        return sign * size * 2.0 ** (scale - 127)

    for r, (c, n) in enumerate(s["rows"]):
        seen = torch.ones(n, c + n, dtype=torch.bool, device="cuda").tril(c).repeat_interleave(g, 0)
        for h in range(hkv):
            q = s["q"][at:at + n, h * g:(h + 1) * g].double().reshape(n * g, d)
            x = (q @ rows("k_cache", r, c + n, h).t() / math.sqrt(d)).masked_fill_(~seen, -math.inf)
            x.sub_(torch.logsumexp(x, -1, keepdim=True)).exp_()
            out[at:at + n, h * g:(h + 1) * g] = (x @ rows("v_cache", r, c + n, h)).view(n, g, d)
        at += n
    return out


def _exact_probs(s):
    vocab, params, row = s["case"]["vocab"], s["params"].double().cpu(), 0
    whole, drafts, first = s["params"].view(torch.int32).cpu(), s["drafts"].long(), 0
    out = torch.empty(s["probs"].shape, dtype=torch.float64, device="cuda")
    place = 2 ** torch.arange(32, device="cuda")
    for r, (h, n) in enumerate(s["rows"]):
        heat, repeat, presence, frequency = params[r, :4].tolist()
        past, prompt = s["history"][r, :h].long(), int(whole[r, 4])
        bias = torch.zeros(vocab, dtype=torch.float64, device="cuda")
        given = {int(t): float(v) for t, v in zip(s["bias_tokens"][r, :int(whole[r, 6])].tolist(), s["bias_values"][r].tolist())}
        if given:
            bias[list(given)] = torch.tensor(list(given.values()), dtype=torch.float64, device="cuda")
        for i in range(n + 1):
            made = torch.cat([past[prompt:], drafts[first:first + i]])
            often = torch.bincount(made, minlength=vocab).double()
            seen = (often > 0) | (torch.bincount(past[:prompt], minlength=vocab) > 0)
            z = s["logits"][row].double()
            z = torch.where(seen, z * torch.where(z > 0, 1.0 / repeat, repeat), z) - (often > 0) * (frequency * often + presence) + bias
            mask = int(s["mask_rows"][row])
            if mask >= 0:
                allowed = ((s["masks"][mask].long()[:, None] & place) != 0).flatten()[:vocab]
                z = z.masked_fill(~allowed, -math.inf)
            if not bool((z > -math.inf).any()):
                out[row] = 0.0
            elif heat > 0:
                out[row] = (z / heat - torch.logsumexp(z / heat, -1)).exp()
            else:
                out[row] = 0.0
                out[row, int((z == z.max()).nonzero()[0])] = 1.0
            row += 1
        first += n
    return out


_exact = {"pages": _exact_pages, "append": _exact_append, "attend": _exact_attend, "probs": _exact_probs}
