"""Cases on which the operators of a drafted (speculative) serving step are measured.

``op`` names the operator:

  "norm_append"    queries and keys normed per head, rotated, keys and values appended to the paged cache
  "latent_append"  one shared latent vector a token normed, its rotary part and the queries' rotated, appended
  "latent"         causal attention over the paged latent cache, absorbed form (queries and outputs in latent space)
  "expanded"       the same attention with keys and values per head expanded from the latents by a weight
  "verify"         drafted tokens accepted or refused against the target's probabilities, and the token after them

Batches are ragged: request r has ``cached`` tokens in front of ``new`` ones.  Lengths come from the case alone
(``lengths_seed``), so that its work does not depend on the inputs' seed.  Pages are shuffled over the cache, an eighth
of them unused.
"""
import math
import random

import numpy as np
import torch

own = False

LATENT, ROPE, NOPE, VALUE = 512, 64, 128, 128  # a latent row is LATENT + ROPE wide; expanded heads NOPE + ROPE and VALUE
ROW = LATENT + ROPE
EPS = 1.0e-6
SCALE = (NOPE + ROPE) ** -0.5


def _batch(name, op, heads, batch, cached, new, **more):
    case = {"name": name, "op": op, "q_heads": heads[0], "kv_heads": heads[1], "batch": batch, "cached_lo": cached[0],
            "cached_hi": cached[1], "new_lo": new[0], "new_hi": new[1], "misses": 0, "miss_lo": 0, "miss_hi": 0,
            "page": 16, "base": 1.0e6, "interleaved": 0, "lengths_seed": 1}
    case.update(more)
    return case


def _heads(name, heads, head_dim, batch, cached, new, **more):
    more = {"head_dim": head_dim, "rotary": head_dim, "cache": "bf16", **more}
    return _batch(name, "norm_append", heads, batch, cached, new, **more)


def _verify(name, batch, vocab, drafts, **more):
    case = {"name": name, "op": "verify", "batch": batch, "vocab": vocab, "drafts_lo": drafts[0], "drafts_hi": drafts[1],
            "given": True, "spread": 3.0, "lengths_seed": 1}
    case.update(more)
    return case


def listed():
    return [
        # next token of 16 users over an 8-bit cache: the launch alone
        _heads("norm_append_users", (28, 4), 128, 16, (1024, 4096), (1, 1), cache="fp8"),
        # a step that mixes cache hits with whole new prompts
        _heads("norm_append_mixed", (32, 8), 128, 64, (512, 8192), (1, 256), misses=32, miss_lo=1024, miss_hi=4096),
        # five drafted tokens of each of 16 users
        _batch("latent_append_users", "latent_append", (16, 1), 16, (1024, 4096), (6, 6)),
        # whole new prompts
        _batch("latent_append_prompts", "latent_append", (32, 1), 32, (0, 0), (1, 1), misses=32, miss_lo=1024, miss_hi=4096),
        # one user's next token: latency
        _batch("latent_user", "latent", (16, 1), 1, (2344, 2344), (1, 1)),
        # next token of 32 users with long contexts, the heads of one of several GPUs
        _batch("latent_decode", "latent", (16, 1), 32, (2048, 8192), (1, 1)),
        # next token with all heads on one GPU
        _batch("latent_decode_wide", "latent", (128, 1), 32, (1024, 4096), (1, 1)),
        # increments of an editor session behind cached prefix and suffix
        _batch("latent_extend", "latent", (28, 1), 32, (2048, 8192), (8, 64)),
        # one user's first prompt, as long as the service's are
        _batch("expanded_prompt", "expanded", (16, 1), 1, (0, 0), (2355, 2355)),
        # whole new prompts, and a long increment behind a cached file
        _batch("expanded_prompts", "expanded", (32, 1), 12, (512, 2048), (200, 700), misses=8, miss_lo=1024, miss_hi=4096),
        # five drafted tokens of one user, a vocabulary of the service's size
        _verify("verify_user", 1, 32004, (5, 5)),
        # up to 15 drafted tokens of 64 users, a large vocabulary of odd size
        _verify("verify_users", 64, 128003, (1, 15)),
    ]


#: what the largest listed case costs, as an estimate that weighs bytes and operations
_MOST = 1.3e-3


def _estimate(case):
    w = work(case)
    return w["bytes"] / 4.0e12 + w["flops"] / 0.6e15


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_append", "latent_append", "latent", "latent", "expanded", "verify"])
    seed = rng.randrange(1, 1 << 20)
    if op == "verify":
        lo = rng.randint(0, 15)
        case = _verify("", _log(rng, 1, 64), _log(rng, 4000, 160000), (lo, rng.randint(max(lo, 1), 15)),
                       given=rng.random() < 0.7, spread=rng.choice([1.0, 3.0]), lengths_seed=seed)
        del case["name"]
        return case
    batch, lo = _log(rng, 1, 64), _log(rng, 64, 8192)
    cached = (lo, min(16384, int(lo * rng.uniform(1.0, 4.0))))
    more = {"page": rng.choice([16, 16, 16, 8, 32, 64, 256]), "base": rng.choice([1.0e4, 5.0e5, 1.0e6]),
            "interleaved": rng.choice([0, 0, 1]), "lengths_seed": seed}
    n = {"latent": _log(rng, 1, 256), "expanded": _log(rng, 128, 2048)}.get(op, _log(rng, 1, 512))
    new = (n, int(n * rng.uniform(1.0, 4.0)))
    if op == "latent" and rng.random() < 0.5:
        new = rng.choice([(1, 1), (1, 16), (6, 6)])
    if op != "latent" and rng.random() < 0.4:
        m = _log(rng, 512, 3000)
        more.update(misses=rng.randint(1, batch), miss_lo=m, miss_hi=min(4096, int(m * rng.uniform(1.0, 2.0))))
    if op == "norm_append":
        heads, head_dim = rng.choice([((32, 8), 128), ((28, 4), 128), ((32, 32), 128), ((4, 4), 64), ((32, 8), 64)])
        case = _heads("", heads, head_dim, batch, cached, new, rotary=rng.choice([head_dim, head_dim, head_dim // 2]),
                      cache=rng.choice(["bf16", "bf16", "fp8"]), **more)
    else:
        heads = rng.choice([(16, 1), (32, 1), (28, 1)] if op == "expanded" else [(16, 1), (32, 1), (28, 1), (128, 1), (4, 1)])
        case = _batch("", op, heads, batch, cached, new, **more)
    del case["name"]
    while _estimate(case) > _MOST:
        case["batch"] = max(1, case["batch"] // 2)
        case["misses"] = min(case["misses"], case["batch"])
        if case["batch"] == 1:
            for key in ("cached_lo", "cached_hi", "new_lo", "new_hi", "miss_lo", "miss_hi"):
                case[key] = -(-case[key] * 3 // 4)
    return case


def _lengths(case):
    """[(cached, new)] of the requests (of "verify": the numbers of drafted tokens), the same for every seed."""
    rng = random.Random(case["lengths_seed"])
    if case["op"] == "verify":
        return [rng.randint(case["drafts_lo"], case["drafts_hi"]) for _ in range(case["batch"])]
    rows = []
    for r in range(case["batch"]):
        if r < case["misses"]:
            rows.append((0, rng.randint(case["miss_lo"], case["miss_hi"])))
        else:
            rows.append((rng.randint(case["cached_lo"], case["cached_hi"]), rng.randint(case["new_lo"], case["new_hi"])))
    rng.shuffle(rows)
    return rows


def work(case):
    rows = _lengths(case)
    if case["op"] == "verify":
        # the target's row behind the last accepted token and, where a token was refused, the draft's there
        # (about seven in ten are accepted); per drafted token two probabilities, an id and a number
        both = sum(1.0 - 0.7 ** n for n in rows) if case["given"] else 0.0
        return {"bytes": int((len(rows) + both) * case["vocab"] * 4 + sum(rows) * 16 + len(rows) * 16), "flops": 0}
    new, hq = sum(n for _, n in rows), case["q_heads"]
    if case["op"] == "norm_append":
        kv = 1 if case["cache"] == "fp8" else 2
        return {"bytes": new * case["head_dim"] * (4 * hq + 2 * case["kv_heads"] * (2 + kv)), "flops": 0}
    if case["op"] == "latent_append":
        return {"bytes": new * (ROW * 4 + ROPE * 4 * hq), "flops": 0}
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in rows)
    keys = sum(c + n for c, n in rows)
    if case["op"] == "latent":
        return {"bytes": keys * ROW * 2 + new * hq * (ROW + LATENT) * 2, "flops": 2 * (ROW + LATENT) * hq * pairs}
    return {"bytes": keys * ROW * 2 + hq * (NOPE + VALUE) * LATENT * 2 + new * hq * (NOPE + ROPE + VALUE) * 2,
            "flops": 2 * (NOPE + ROPE + VALUE) * hq * pairs + 2 * keys * hq * (NOPE + VALUE) * LATENT}


# --- inputs ------------------------------------------------------------------------------------------------------------


def _pages(case, rows, seed):
    """(block table, pages) with disjoint pages in an order drawn from the seed."""
    need = [-(-(c + n) // case["page"]) for c, n in rows]
    pages = sum(need) + max(2, sum(need) // 8)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(rows), max(need)), int(order[-1]), dtype=torch.int32)
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = order[at:at + k]
        at += k
    return table.cuda(), pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = _lengths(case)
    state = {"case": case, "rows": rows}

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        return torch.randn(shape, dtype=dtype, device="cuda", generator=gen).mul_(scale)

    if case["op"] == "verify":
        return _prepare_verify(case, gen, rows, state)
    cached, new = [c for c, _ in rows], [n for _, n in rows]
    total, hq, hkv, page = sum(new), case["q_heads"], case["kv_heads"], case["page"]
    table, pages = _pages(case, rows, seed)
    # request and position of every new token: what an engine's step has at hand
    state["table"] = table
    state["req"] = torch.repeat_interleave(torch.arange(len(rows)), torch.tensor(new)).cuda()
    state["pos"] = torch.cat([torch.arange(c, c + n) for c, n in rows]).cuda()
    width = case["rotary"] if case["op"] == "norm_append" else ROPE
    state["inv_freq"] = case["base"] ** (-2.0 * np.arange(width // 2) / width)
    if case["op"] == "norm_append":
        d = case["head_dim"]
        # activations in front of a norm have scales of their own for each head
        state["q"] = normal(total, hq, d) * torch.linspace(0.3, 3.0, hq, device="cuda").to(torch.bfloat16)[:, None]
        state["k"], state["v"] = normal(total, hkv, d, scale=2.0), normal(total, hkv, d)
        state["q_weight"], state["k_weight"] = normal(d, scale=0.2) + 1.0, normal(d, scale=0.2) + 1.0
        shape = (pages, hkv, page, d)
        state["scale"] = 6.0 / 448.0  # what a normed and weighted element seldom passes reaches the largest code
        for name in ("k_cache", "v_cache"):
            state[name] = normal(*shape)
            if case["cache"] == "fp8":
                codes = torch.empty(shape, dtype=torch.uint8, device="cuda")
                for part, to in zip(state[name].split(4096), codes.split(4096)):
                    to.copy_((part.float() / state["scale"]).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
                state[name] = codes
        if own:
            state["q_out"] = torch.empty_like(state["q"])
    else:
        d = ROW
        cache = normal(pages, page, ROW)
        state["cache"] = cache
        if case["op"] == "latent_append":
            state["q"] = normal(total, hq, NOPE + ROPE)
            state["kv"] = normal(total, ROW, scale=2.0)
            state["weight"] = normal(LATENT, scale=0.2) + 1.0
            if own:
                state["q_out"] = torch.empty(total, hq, ROPE, dtype=torch.bfloat16, device="cuda")
        elif case["op"] == "latent":
            state["q"] = normal(total, hq, ROW)
            if own:
                state["out"] = torch.empty(total, hq, LATENT, dtype=torch.bfloat16, device="cuda")
        else:
            state["q"] = normal(total, hq, NOPE + ROPE)
            state["w_kv"] = normal(hq, NOPE + VALUE, LATENT, scale=LATENT ** -0.5)
            if own:
                state["out"] = torch.empty(total, hq, VALUE, dtype=torch.bfloat16, device="cuda")
    if own:
        from paper_2505_21889_amd import binding as E
        state["batch"] = E.BatchDesc(cached, new, table, hq, hkv, d, page, pages)
        if case["op"] in ("latent", "expanded"):
            size = E.efim_latent_workspace_bytes if case["op"] == "latent" else E.efim_latent_expanded_workspace_bytes
            state["ws_bytes"] = size(state["batch"])
            state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device="cuda")
    return state


def _prepare_verify(case, gen, rows, state):
    vocab, drafts = case["vocab"], sum(rows)
    first = np.concatenate([[0], np.cumsum(rows)])  # first drafted token of each request; its first target row is r further on
    state["first"] = torch.from_numpy(first[:-1].astype(np.int64)).cuda()
    state["count"] = torch.tensor(rows, dtype=torch.int64, device="cuda")
    target = torch.empty(drafts + len(rows), vocab, device="cuda")
    draft = torch.empty(drafts, vocab, device="cuda")
    tokens = torch.empty(drafts, dtype=torch.int32, device="cuda")

    def probabilities(logits):
        p = torch.softmax(logits, -1)
        p[p < 1.0e-8] = 0.0  # engines cut the tail
        return p.div_(p.sum(-1, keepdim=True))

    for r, n in enumerate(rows):
        logits = torch.randn(n + 1, vocab, device="cuda", generator=gen).mul_(case["spread"])
        t0, d0 = int(first[r]) + r, int(first[r])
        target[t0:t0 + n + 1] = probabilities(logits)
        if n:
            near = logits[:n] + torch.randn(n, vocab, device="cuda", generator=gen).mul_(0.5)
            draft[d0:d0 + n] = probabilities(near)
            # without probabilities of its own a draft proposes the likeliest token
            tokens[d0:d0 + n] = (torch.multinomial(draft[d0:d0 + n], 1, generator=gen)[:, 0] if case["given"] else near.argmax(-1)).int()
    state.update(target=target, draft=draft if case["given"] else None, tokens=tokens,
                 uniforms=torch.rand(drafts + len(rows), device="cuda", generator=gen))
    if own:
        from paper_2505_21889_amd import binding as E
        state["drafts"] = np.asarray(rows, dtype=np.int32)
        state["out"] = torch.empty(drafts + len(rows), dtype=torch.int32, device="cuda")
        state["accepted"] = torch.empty(len(rows), dtype=torch.int32, device="cuda")
        state["ws_bytes"] = E.efim_verify_workspace_bytes(len(rows), vocab)
        state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device="cuda")
    return state


# --- the operators -------------------------------------------------------------------------------------------------------


def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _own_norm_append(s):
    from paper_2505_21889_amd import binding as E
    case = s["case"]
    common = (s["batch"], s["q"], s["q_out"], s["k"], s["v"], s["q_weight"], s["k_weight"], EPS, s["k_cache"], s["v_cache"],
              s["inv_freq"], case["rotary"], case["interleaved"])
    if case["cache"] == "fp8":
        E.efim_norm_rope_append_fp8(*common, s["scale"], s["scale"])
    else:
        E.efim_norm_rope_append(*common)
    return _appended(s, s["q_out"])


def _appended(s, q):
    kind = torch.float8_e4m3fn if s["case"]["cache"] == "fp8" else torch.bfloat16
    return {"q": q, "k_cache": s["k_cache"].view(kind), "v_cache": s["v_cache"].view(kind)}


def _own_latent_append(s):
    from paper_2505_21889_amd import binding as E
    E.efim_latent_append(s["batch"], s["q"][:, :, NOPE:], NOPE + ROPE, s["q_out"], ROPE, s["kv"], ROW, s["weight"], EPS,
                         s["cache"], s["inv_freq"], s["case"]["interleaved"])
    return {"q": s["q_out"], "cache": s["cache"]}


def _own_latent(s):
    from paper_2505_21889_amd import binding as E
    E.efim_latent_attention(s["batch"], s["q"], s["cache"], s["out"], SCALE, s["ws"], s["ws_bytes"])
    return s["out"]


def _own_expanded(s):
    from paper_2505_21889_amd import binding as E
    E.efim_latent_attention_expanded(s["batch"], s["q"], s["cache"], s["w_kv"], s["out"], SCALE, s["ws"], s["ws_bytes"])
    return s["out"]


def _own_verify(s):
    from paper_2505_21889_amd import binding as E
    vocab = s["case"]["vocab"]
    E.efim_verify_drafts(s["drafts"], vocab, s["target"], vocab, s["draft"], vocab, s["tokens"], s["uniforms"], s["out"],
                         s["accepted"], s["ws"], s["ws_bytes"])
    return {"tokens": s["out"], "accepted": s["accepted"]}


_run_own = {"norm_append": _own_norm_append, "latent_append": _own_latent_append, "latent": _own_latent,
            "expanded": _own_expanded, "verify": _own_verify}


def _rms(x, weight):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()


def _rotate(x, s):
    """Rotates the leading elements of float rows [T, heads, d] at the tokens' positions."""
    # (angles in 64 bits: of a position in the ten thousands 32 bits keep three digits of the angle)
    angle = s["pos"].double()[:, None] * torch.from_numpy(s["inv_freq"]).cuda()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    half = cos.shape[-1]
    y = x.clone()
    if s["case"]["interleaved"]:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    return y


def _slots(s):
    page = s["case"]["page"]
    return s["table"][s["req"], s["pos"] // page].long(), s["pos"] % page


def _plain_norm_append(s):
    at, slot = _slots(s)
    k, v = _rotate(_rms(s["k"], s["k_weight"]), s).to(torch.bfloat16), s["v"]
    if s["case"]["cache"] == "fp8":
        k, v = (x.float().div_(s["scale"]).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, v))
    s["k_cache"][at, :, slot] = k
    s["v_cache"][at, :, slot] = v
    return _appended(s, _rotate(_rms(s["q"], s["q_weight"]), s).to(torch.bfloat16))


def _plain_latent_append(s):
    at, slot = _slots(s)
    kv = s["kv"]
    s["cache"][at, slot, :LATENT] = _rms(kv[:, :LATENT], s["weight"]).to(torch.bfloat16)
    s["cache"][at, slot, LATENT:] = _rotate(kv[:, None, LATENT:].float(), s)[:, 0].to(torch.bfloat16)
    return {"q": _rotate(s["q"][:, :, NOPE:].float(), s).to(torch.bfloat16), "cache": s["cache"]}


def _requests(s):
    """(first new row, rows, cached keys, latent rows [keys, ROW] in 32 bits) of every request with new tokens."""
    at, page = 0, s["case"]["page"]
    for r, (c, n) in enumerate(s["rows"]):
        if n:
            yield at, n, c, s["cache"][s["table"][r, :-(-(c + n) // page)].long()].view(-1, ROW)[:c + n].float()
        at += n


def _weights(scores, c, n):
    """Softmax over the visible keys of scores [..., n, keys] whose row i sees c + i + 1."""
    hidden = torch.arange(c + n, device="cuda") > torch.arange(c, c + n, device="cuda")[:, None]
    scores.masked_fill_(hidden, -math.inf)
    scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    return scores.div_(scores.sum(-1, keepdim=True))


def _plain_latent(s):
    out = torch.empty(s["q"].shape[:2] + (LATENT,), dtype=torch.bfloat16, device="cuda")
    for at, n, c, latent in _requests(s):
        q = s["q"][at:at + n].float().transpose(0, 1).reshape(-1, ROW)  # heads outermost
        p = _weights((q @ latent.T).mul_(SCALE).view(-1, n, c + n), c, n)
        out[at:at + n] = (p.view(-1, c + n) @ latent[:, :LATENT]).view(-1, n, LATENT).transpose(0, 1)
    return out


def _plain_expanded(s):
    hq = s["case"]["q_heads"]
    w = s["w_kv"].float().view(-1, LATENT)
    out = torch.empty(s["q"].shape[:2] + (VALUE,), dtype=torch.bfloat16, device="cuda")
    for at, n, c, latent in _requests(s):
        kv = (latent[:, :LATENT] @ w.T).view(c + n, hq, NOPE + VALUE).transpose(0, 1)
        rope = latent[:, LATENT:].expand(hq, -1, -1)
        keys = torch.cat([kv[..., :NOPE], rope], -1).transpose(1, 2).contiguous()
        scores = torch.bmm(s["q"][at:at + n].float().transpose(0, 1).contiguous(), keys).mul_(SCALE)
        out[at:at + n] = torch.bmm(_weights(scores, c, n), kv[..., NOPE:].contiguous()).transpose(0, 1)
    return out


def _fixed(p):
    """Probabilities as whole numbers of 2^-40, what is no number as zero."""
    return (torch.nan_to_num(p, nan=0.0).clamp(0.0, 1.0) * 2.0 ** 40).long()


def _plain_verify(s):
    target, draft, tokens, u = s["target"], s["draft"], s["tokens"].long(), s["uniforms"]
    first, count = s["first"], s["count"]
    req = torch.repeat_interleave(torch.arange(len(count), device="cuda"), count, output_size=len(tokens))
    own_row = torch.arange(len(tokens), device="cuda")
    p = target[own_row + req, tokens].double()
    q = draft[own_row, tokens].double() if draft is not None else 1.0
    refused = ~(u[own_row + req].double() * q < p)  # (the product of two 32-bit numbers is exact in 64)
    # the first refused token of each request
    at = torch.where(refused, own_row - first[req], count[req])
    accepted = count.clone().scatter_reduce_(0, req, at, "amin")
    weight = _fixed(target[first + torch.arange(len(count), device="cuda") + accepted])
    rejected = (accepted < count)[:, None]
    whole = weight
    if len(tokens):
        row = torch.minimum(first + accepted, torch.full_like(first, len(tokens) - 1))
        if draft is not None:
            other = _fixed(draft[row])
        else:
            other = torch.zeros_like(weight).scatter_(1, tokens[row][:, None], 1 << 40)
        weight = torch.where(rejected, (weight - other).clamp_(min=0), weight)
    weight = torch.where(weight.sum(-1, keepdim=True) == 0, whole, weight)
    total = weight.sum(-1)
    part = (u[first + torch.arange(len(count), device="cuda") + count] * 2.0 ** 24).long().clamp(0, 2 ** 24 - 1)
    below = part * (total >> 24) + ((part * (total & (2 ** 24 - 1))) >> 24)  # floor(u total), u in units of 2^-24
    token = (weight.cumsum(-1) <= below[:, None]).sum(-1)
    token = torch.where(total == 0, torch.full_like(token, -1), token)
    out = torch.full((len(u),), -1, dtype=torch.int32, device="cuda")
    out[own_row + req] = torch.where(own_row - first[req] < accepted[req], tokens, -1).int()
    out[first + torch.arange(len(count), device="cuda") + accepted] = token.int()
    return {"tokens": out, "accepted": accepted.int()}


_run_plain = {"norm_append": _plain_norm_append, "latent_append": _plain_latent_append, "latent": _plain_latent,
              "expanded": _plain_expanded, "verify": _plain_verify}


# --- the definitions in 64 bits ------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return _exact[case["op"]](s)


def _turned(x, s):
    """Rows [T, heads, d] in 64 bits, pairs taken as complex numbers and multiplied by exp(i angle)."""
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["pos"].double()[:, None] * torch.from_numpy(s["inv_freq"]).cuda())[:, None]
    half = turn.shape[-1]
    lead = x[..., :2 * half].unflatten(-1, (half, 2) if s["case"]["interleaved"] else (2, half))
    if not s["case"]["interleaved"]:
        lead = lead.transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(lead.contiguous()) * turn)
    if not s["case"]["interleaved"]:
        z = z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), x[..., 2 * half:]], -1)


def _normed(x, weight):
    x = x.double()
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()


def _exact_norm_append(s):
    case, at, parts = s["case"], 0, {}
    parts["q"] = _turned(_normed(s["q"], s["q_weight"]), s)
    fp8 = case["cache"] == "fp8"
    for name, new in (("k", _turned(_normed(s["k"], s["k_weight"]), s)), ("v", s["v"].double())):
        cache = s[name + "_cache"]
        cache = (cache.view(torch.float8_e4m3fn) if fp8 else cache).double()
        if fp8:
            new = (new / s["scale"]).clamp(-448, 448)
        at = 0
        for r, (c, n) in enumerate(s["rows"]):  # token by token of a request, page by page
            where = torch.arange(c, c + n, device="cuda")
            flat = s["table"][r].long()[where.div(case["page"], rounding_mode="floor")]
            cache[flat, :, where.remainder(case["page"])] = new[at:at + n]
            at += n
        parts[name + "_cache"] = cache
    return parts


def _exact_latent_append(s):
    case, at = s["case"], 0
    new = torch.cat([_normed(s["kv"][:, :LATENT], s["weight"]), _turned(s["kv"][:, None, LATENT:].double(), s)[:, 0]], -1)
    cache = s["cache"].double()
    for r, (c, n) in enumerate(s["rows"]):
        where = torch.arange(c, c + n, device="cuda")
        cache[s["table"][r].long()[where.div(case["page"], rounding_mode="floor")], where.remainder(case["page"])] = new[at:at + n]
        at += n
    return {"q": _turned(s["q"][:, :, NOPE:].double(), s), "cache": cache}


def _exact_rows(s):
    at = 0
    for r, (c, n) in enumerate(s["rows"]):
        where = torch.arange(c + n, device="cuda")
        page = s["case"]["page"]
        yield at, c, n, s["cache"][s["table"][r].long()[where.div(page, rounding_mode="floor")], where.remainder(page)].double()
        at += n


def _exact_softmax(x, c):
    """softmax of [n, keys] where row i sees the keys 0 .. c + i, through the logarithm of the sum."""
    n, keys = x.shape
    seen = torch.ones(n, keys, dtype=torch.bool, device="cuda").tril(c)
    x = x.where(seen, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
    return (x - torch.logsumexp(x, -1, keepdim=True)).exp()


def _exact_latent(s):
    out = torch.empty(s["q"].shape[:2] + (LATENT,), dtype=torch.float64, device="cuda")
    for at, c, n, rows in _exact_rows(s):
        for h in range(s["case"]["q_heads"]):
            x = s["q"][at:at + n, h].double() @ rows.t() * SCALE
            out[at:at + n, h] = _exact_softmax(x, c) @ rows[:, :LATENT]
    return out


def _exact_expanded(s):
    out = torch.empty(s["q"].shape[:2] + (VALUE,), dtype=torch.float64, device="cuda")
    for at, c, n, rows in _exact_rows(s):
        for h in range(s["case"]["q_heads"]):
            up, q = s["w_kv"][h].double(), s["q"][at:at + n, h].double()
            # the query meets the latent itself, the values are expanded behind the sum
            x = (q[:, :NOPE] @ up[:NOPE] @ rows[:, :LATENT].t() + q[:, NOPE:] @ rows[:, LATENT:].t()) * SCALE
            out[at:at + n, h] = _exact_softmax(x, c) @ rows[:, :LATENT] @ up[NOPE:].t()
    return out


def _exact_verify(s):
    target, tokens, u = s["target"].cpu().numpy(), s["tokens"].cpu().numpy(), s["uniforms"].cpu().numpy()
    draft = None if s["draft"] is None else s["draft"].cpu().numpy()
    out, accepted, d, t = np.full(len(u), -1, np.int32), np.zeros(len(s["rows"]), np.int32), 0, 0

    def whole(row):
        return np.floor(np.clip(np.nan_to_num(row, nan=0.0), 0.0, 1.0).astype(np.float64) * 2.0 ** 40).astype(np.int64)

    for r, n in enumerate(s["rows"]):
        a = 0
        while a < n and float(u[t + a]) * (1.0 if draft is None else float(draft[d + a, tokens[d + a]])) < float(target[t + a, tokens[d + a]]):
            out[t + a] = tokens[d + a]
            a += 1
        weight = p = whole(target[t + a])
        if a < n:
            if draft is None:
                weight = p.copy()
                weight[tokens[d + a]] = max(0, int(p[tokens[d + a]]) - (1 << 40))
            else:
                weight = np.maximum(p - whole(draft[d + a]), 0)
            if not weight.any():
                weight = p
        total = int(weight.sum())
        below = (min(int(float(u[t + n]) * 2 ** 24), 2 ** 24 - 1) * total) >> 24
        out[t + a] = int(np.searchsorted(np.cumsum(weight), below, side="right")) if total else -1
        accepted[r] = a
        d, t = d + n, t + n + 1
    return {"tokens": torch.from_numpy(out), "accepted": torch.from_numpy(accepted)}


_exact = {"norm_append": _exact_norm_append, "latent_append": _exact_latent_append, "latent": _exact_latent,
          "expanded": _exact_expanded, "verify": _exact_verify}
