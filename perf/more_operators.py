"""Cases of further operators for serving a language model over a ragged batch: a paged key-value cache held in 8 bits with a
scale for each block of tokens and head (quantised as it is written, read back in 16 bits, attention of one new token over it), and
layers that keep a state under the gated delta rule (packed prompts, single tokens).

``run`` computes a case in its plain form (elementary torch operations in 32 bits) or, with ``own`` set, through the
package's entry points; ``exact`` computes it from the operator's definition in 64 bits.

The 8-bit cache.  A code stands for code * scale[block, head].  int8: scale is the block's largest magnitude / 127, rounded up to 11
significant bits; a code is x / scale rounded to the nearest whole number, halves away from zero.  e4m3: scale is the smallest power of two that
brings the largest magnitude to 448 or less; a code is x / scale rounded to the nearest e4m3 value, halves to even.  Inputs and scales have
11 bits at most, so that a quotient that is no half is at least 2^-19 of itself away from one, and a rounded division decides rightly.
A block whose first place is written is begun anew; one that is continued keeps its scale where the new tokens fit, else the codes that it holds
are converted to the new one.
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
_TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
_CHUNK = 64


# ---------------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the keys and values of one decoding step, and the blocks they went to as 16-bit values
        {"name": "append_read_decode_255", "op": "append_read", "nreq": 255, "hq": 32, "hkv": 8, "d": 128, "block": 16, "most": 4096, "law": "decode",
         "type": "bf16", "cache": "int8"},
        # a batch of prompts, some of which continue a cached part: written, then read back for the prompts' own attention
        {"name": "append_read_prompts_48", "op": "append_read", "nreq": 48, "hq": 16, "hkv": 8, "d": 128, "block": 64, "most": 2500, "law": "prompts",
         "type": "f16", "cache": "e4m3"},
        # the cached prefix of one short conversation
        {"name": "read_prefix_1000", "op": "read", "nreq": 1, "hkv": 4, "d": 80, "block": 16, "most": 1000, "law": "same", "type": "f16", "cache": "e4m3"},
        # the prefixes of a batch whose prompts go on
        {"name": "read_prefixes_32", "op": "read", "nreq": 32, "hkv": 8, "d": 128, "block": 32, "most": 8192, "law": "uniform", "type": "bf16", "cache": "int8"},
        # a single user's short context: latency
        {"name": "attention_one_777", "op": "attention", "nreq": 1, "hq": 8, "hkv": 2, "d": 64, "block": 16, "most": 777, "law": "same", "window": 0,
         "type": "f16", "cache": "int8"},
        # an ordinary serving batch, lengths from 0 to 4096, grouped heads
        {"name": "attention_batch_64", "op": "attention", "nreq": 64, "hq": 32, "hkv": 8, "d": 128, "block": 16, "most": 4096, "law": "uniform", "window": 0,
         "type": "bf16", "cache": "int8"},
        # a few very long contexts, the ones that an 8-bit cache is for
        {"name": "attention_long_131072", "op": "attention", "nreq": 4, "hq": 32, "hkv": 8, "d": 128, "block": 64, "most": 131072, "law": "same", "window": 0,
         "type": "bf16", "cache": "e4m3"},
        # a few short prompts of a small model
        {"name": "delta_prompts_short", "op": "delta", "nseq": 4, "tokens": 333, "hk": 4, "rep": 1, "dk": 64, "dv": 64, "state": False},
        # an ordinary batch of prompts that continue a state, two value heads to a key head
        {"name": "delta_prompts_batch", "op": "delta", "nseq": 16, "tokens": 32768, "hk": 8, "rep": 2, "dk": 128, "dv": 128, "state": True},
        # one long prompt: a chain of a thousand chunks
        {"name": "delta_prompt_long", "op": "delta", "nseq": 1, "tokens": 65536, "hk": 16, "rep": 1, "dk": 128, "dv": 128, "state": False},
        # one token of one user
        {"name": "delta_step_1", "op": "delta_step", "nreq": 1, "hk": 16, "rep": 1, "dk": 128, "dv": 128, "type": "f16"},
        # one token each of a busy server's requests: the states are the traffic
        {"name": "delta_step_256", "op": "delta_step", "nreq": 256, "hk": 8, "rep": 2, "dk": 128, "dv": 128, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append_read", "append_read", "read", "attention", "attention", "delta", "delta", "delta_step"])
    if op in ("append_read", "read"):
        hkv, d = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 80, 96, 128, 256])
        case = {"op": op, "nreq": _log(rng, 1, 512), "hkv": hkv, "d": d, "block": rng.choice([8, 16, 32, 48, 64, 128]), "type": rng.choice(["bf16", "f16"]),
                "cache": rng.choice(["int8", "e4m3"])}
        fit = max(16, (1 << 26) // (case["nreq"] * hkv * d))             # values of the keys, all requests at their longest
        if op == "read":
            return {**case, "most": _log(rng, 8, min(65536, fit)), "law": rng.choice(["same", "uniform", "skewed"])}
        case["law"] = rng.choice(["decode", "prompts"])
        return {**case, "hq": hkv * rng.choice([1, 2, 4]), "most": _log(rng, 8, 4096 if case["law"] == "decode" else min(65536, fit))}
    if op == "attention":
        hkv, d = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 128, 256])
        nreq = _log(rng, 1, 256)
        most = _log(rng, 16, max(32, min(131072, (1 << 29) // (nreq * hkv * d))))
        return {"op": op, "nreq": nreq, "hq": hkv * rng.choice([1, 2, 4, 6, 8, 16]), "hkv": hkv, "d": d, "block": rng.choice([8, 16, 32, 48, 64, 128]),
                "most": most, "law": rng.choice(["same", "uniform", "skewed"]), "window": rng.choice([0, 0, 0, max(1, most // 3)]),
                "type": rng.choice(["bf16", "f16"]), "cache": rng.choice(["int8", "e4m3"])}
    if op == "delta":
        hk, rep, dk, dv = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2]), rng.choice([64, 96, 128]), rng.choice([64, 80, 128])
        return {"op": op, "nseq": _log(rng, 1, 64), "tokens": _log(rng, 64, 65536), "hk": hk, "rep": rep, "dk": dk, "dv": dv, "state": rng.random() < 0.5}
    return {"op": op, "nreq": _log(rng, 1, 256), "hk": rng.choice([1, 3, 4, 8]), "rep": rng.choice([1, 2]), "dk": rng.choice([32, 64, 128]),
            "dv": rng.choice([64, 96, 128]), "type": rng.choice(["bf16", "f16"])}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 29)
    return g


def _normal(g, shape, dtype=torch.float32, std=1.0):
    x = torch.empty(shape, dtype=torch.float32, device="cuda")
    return x.normal_(0.0, std, generator=g).to(dtype)


def _device(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _lengths(rng, n, most, law):
    """Lengths in any order; their law is the same for every seed, so that every seed fills a batch alike."""
    if law == "same":
        return [most] * n
    if law == "uniform":
        lens = [i * most // max(1, n - 1) for i in range(n)]
        rng.shuffle(lens)
        return lens
    lens = [1 + i * (max(1, most // 16) - 1) // max(1, n - 1) for i in range(n)]      # skewed: one long context beside many short ones
    rng.shuffle(lens)
    lens[n // 2] = most
    return lens


def _table(rng, pages, width, ids):
    """Row r: pages[r] of the ids, in order; 0 behind them."""
    at, rows = 0, []
    for p in pages:
        rows.append(ids[at:at + p] + [0] * (width - p))
        at += p
    return _device(rows).reshape(len(pages), width)


def _scale_of(amax, top):
    """The scale of values up to amax (0 for those that are taken for zero)."""
    x, e = torch.frexp(amax / top)
    x = torch.ceil(x * 2048) / 2048 if top == 127.0 else torch.where(x > 0.5, 1.0, 0.5)
    return torch.where(amax < 2.0 ** -100, 0.0, torch.ldexp(x, e))


def _codes(x, scale, top):
    y = torch.where(scale > 0, x / torch.where(scale > 0, scale, 1.0), 0.0)
    if top == 127.0:
        return (torch.sign(y) * torch.floor(y.abs() + 0.5)).to(torch.int8)
    return y.to(torch.float8_e4m3fn)


def _cache(g, blocks, block, hkv, d, dtype):
    """A cache in use: every block holds values of its own magnitude, columns of very different ones (as keys have)."""
    x = _normal(g, (blocks, block, hkv, d)) * torch.exp(_normal(g, (hkv, d)) * 0.7)
    x = x.to(torch.bfloat16).float()
    scale = _scale_of(x.abs().amax((1, 3)), _TOP[dtype])
    return _codes(x, scale[:, None, :, None], _TOP[dtype]), scale.contiguous()


def prepare(case, seed):
    g, rng, op = _generator(seed), random.Random(1000003 * int(seed) + 31), case["op"]
    if op == "append_read":
        n, hq, hkv, d, block, most, dt, ct = (case[x] for x in ("nreq", "hq", "hkv", "d", "block", "most", "type", "cache"))
        if case["law"] == "decode":     # every request grows by a token; the pool holds the blocks that they grow into
            past, new = [rng.randrange(most) for _ in range(n)], [1] * n
        else:       # a third of the requests continue; an eighth of all have nothing to add in this step
            past = [rng.randrange(most + 1) if rng.random() < 1 / 3 else 0 for _ in range(n)]
            new = [0 if i % 8 == 7 else 1 + i * (most - 1) // max(1, n - 1) for i in range(n)]
            rng.shuffle(new)
        pages = [(a + b + block - 1) // block for a, b in zip(past, new)]
        fresh = [p - a // block if b else 0 for a, b, p in zip(past, new, pages)]       # blocks that the call writes to
        blocks = 1 + sum((b + block - 2) // block + 1 if b else 0 for b in new)         # the most that any seed needs, and a last one that is nobody's
        ids = list(range(blocks - 1))
        rng.shuffle(ids)
        rows, at, width = [], 0, (2 * most + block - 1) // block + 1
        for p, f in zip(pages, fresh):                                                  # (blocks in front of those are not looked at)
            rows.append([0] * (p - f) + ids[at:at + f] + [0] * (width - p))
            at += f
        off = [0]
        for b in new:
            off.append(off[-1] + b)
        tokens = off[-1]
        qkv = _normal(g, (tokens + 3, hq + 2 * hkv, d)) * torch.exp(_normal(g, (hq + 2 * hkv, d)) * 0.7)
        qkv = qkv.to(_TYPES[dt])                        # the fused projection's output, padded: k and v are views into it
        cache, scale = zip(*(_cache(g, blocks, block, hkv, d, _TYPES[ct]) for _ in range(2)))
        return {"op": op, "k": qkv[:, hq:hq + hkv], "v": qkv[:, hq + hkv:], "tokens": tokens, "offsets": _device(off),
                "total": _device([a + b for a, b in zip(past, new)]), "table": _device(rows).reshape(n, width), "cache": cache, "scale": scale,
                "all": torch.arange(blocks, dtype=torch.int32, device="cuda")[None], "ends": _device([0, blocks * block])}
    if op == "read":
        n, hkv, d, block, most, ct = (case[x] for x in ("nreq", "hkv", "d", "block", "most", "cache"))
        lens = _lengths(rng, n, most, case["law"])
        pages = [(x + block - 1) // block for x in lens]
        blocks = sum(pages) + 3
        ids = list(range(blocks))
        rng.shuffle(ids)
        off = [0]
        for x in lens:
            off.append(off[-1] + x)
        cache, scale = zip(*(_cache(g, blocks, block, hkv, d, _TYPES[ct]) for _ in range(2)))
        return {"op": op, "cache": cache, "scale": scale, "table": _table(rng, pages, max(pages + [1]), ids), "offsets": _device(off), "tokens": off[-1],
                "type": _TYPES[case["type"]]}
    if op == "attention":
        n, hq, hkv, d, block, most, dt, ct = (case[x] for x in ("nreq", "hq", "hkv", "d", "block", "most", "type", "cache"))
        lens = _lengths(rng, n, most, case["law"])
        pages = [(x + block - 1) // block for x in lens]
        blocks = sum(pages) + 5
        ids = list(range(blocks))
        rng.shuffle(ids)
        cache, scale = zip(*(_cache(g, blocks, block, hkv, d, _TYPES[ct]) for _ in range(2)))
        return {"op": op, "q": _normal(g, (n, hq, d), _TYPES[dt], 0.7), "cache": cache, "scale": scale, "table": _table(rng, pages, max(pages + [1]), ids),
                "lens": _device(lens), "window": case["window"], "sm_scale": d ** -0.5}
    hk, dk, dv = case["hk"], case["dk"], case["dv"]
    h = hk * case["rep"]
    unit = lambda x: x * torch.rsqrt(x.square().sum(-1, keepdim=True) + 1e-6)           # noqa: E731  queries and keys are normalised
    # heads that forget fast and heads that forget slowly, by an amount that each token chooses
    rate = torch.exp2(-torch.linspace(0, 8, h, device="cuda"))
    gate = lambda m: (-rate * torch.log1p(torch.exp(_normal(g, (m, h)))), torch.sigmoid(_normal(g, (m, h))))      # noqa: E731
    if op == "delta":
        t, n = case["tokens"], case["nseq"]
        cuts = [0] + sorted(rng.randrange(t + 1) for _ in range(n - 1)) + [t]
        decay, beta = gate(t)
        bf = torch.bfloat16
        return {"op": op, "q": unit(_normal(g, (t, hk, dk))).to(bf), "k": unit(_normal(g, (t, hk, dk))).to(bf), "v": _normal(g, (t, h, dv), bf),
                "decay": decay, "beta": beta, "sm_scale": dk ** -0.5, "offsets": _device(cuts), "most": max(b - a for a, b in zip(cuts, cuts[1:])),
                "state": _normal(g, (n, h, dk, dv), std=0.3) if case["state"] else None}
    n, dt = case["nreq"], _TYPES[case["type"]]
    pool = n + n // 4 + 1
    decay, beta = gate(n)
    return {"op": op, "q": unit(_normal(g, (n, hk, dk))).to(dt), "k": unit(_normal(g, (n, hk, dk))).to(dt), "v": _normal(g, (n, h, dv), dt), "decay": decay,
            "beta": beta, "sm_scale": dk ** -0.5, "state": _normal(g, (pool, h, dk, dv), std=0.3), "state_out": torch.zeros(pool, h, dk, dv, device="cuda"),
            "at": torch.randperm(pool, generator=g, device="cuda")[:n].to(torch.int32)}


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plain_append(s, x, cache, scale):
    block, top, tokens = cache.shape[1], _TOP[cache.dtype], s["tokens"]
    off, total, table = s["offsets"].long(), s["total"].long(), s["table"].long()
    past, spare = total - (off[1:] - off[:-1]), cache.shape[0] - 1
    t = torch.arange(tokens, device=off.device)
    r = torch.searchsorted(off[1:], t, right=True)
    p = past[r] + t - off[r]
    at, place = table[r, p // block], p % block
    x = x[:tokens].float()
    amax = torch.zeros_like(scale).scatter_reduce(0, at[:, None].expand(-1, scale.shape[1]), x.abs().amax(-1), "amax")
    # the block that a request continues: its first one, where that holds tokens
    goes_on = (total > past) & (past % block > 0)
    held = torch.where(goes_on, table[torch.arange(total.numel(), device=off.device), past // block], spare)
    went_on = torch.zeros(scale.shape[0], dtype=torch.bool, device=off.device).index_fill(0, held, True)[:, None]
    old = torch.where(went_on, scale, 0.0)
    new = torch.where(amax > old * top, _scale_of(amax, top), old)
    rows = cache[held].float() * old[held][:, None, :, None]
    grows = goes_on[:, None] & (new[held] > old[held])
    change = grows[:, None, :, None] & (torch.arange(block, device=off.device)[None, :] < (past % block)[:, None])[:, :, None, None]
    cache[held] = torch.where(change, _codes(rows, new[held][:, None, :, None], top).float(), cache[held].float()).to(cache.dtype)
    cache[at, place] = _codes(x, new[at][:, :, None], top)
    touched = torch.zeros(scale.shape[0], dtype=torch.bool, device=off.device).index_fill(0, at, True)[:, None]
    scale.copy_(torch.where(touched, new, scale))


def _plain_append_read(s):
    out = {}
    for name, x, cache, scale in zip("kv", (s["k"], s["v"]), s["cache"], s["scale"]):
        _plain_append(s, x, cache, scale)
        out[name] = (cache.float() * scale[:, None, :, None]).flatten(0, 1).to(x.dtype)
        out[name + "_scale"] = scale
    return out


def _plain_read(s):
    off, table = s["offsets"].long(), s["table"].long()
    t = torch.arange(s["tokens"], device=off.device)
    r = torch.searchsorted(off[1:], t, right=True)
    p, block = t - off[r], s["cache"][0].shape[1]
    at, place = table[r, p // block], p % block
    return {name: (c[at, place].float() * w[at][:, :, None]).to(s["type"]) for name, c, w in zip("kv", s["cache"], s["scale"])}


def _plain_attention(s):
    q, table, lens = s["q"].float(), s["table"].long(), s["lens"].long()
    n, hq, d = q.shape
    kv = [(c[table].float() * w[table][:, :, None, :, None]).flatten(1, 2) for c, w in zip(s["cache"], s["scale"])]      # [request, token, head, d]
    hkv = kv[0].shape[2]
    at = torch.arange(kv[0].shape[1], device=q.device)[None, :]
    on = at < lens[:, None]
    if s["window"]:
        on = on & (at >= lens[:, None] - s["window"])
    x = s["sm_scale"] * torch.einsum("nhgd,nthd->nhgt", q.view(n, hkv, hq // hkv, d), kv[0])
    x = torch.where(on[:, None, None, :], x, -torch.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)                              # (a request of no tokens has only -inf)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = torch.einsum("nhgt,nthd->nhgd", p, kv[1]) / total.clamp(min=1e-38)
    lse = torch.where(total > 0, top + torch.log(total), -torch.inf)
    return {"out": out.reshape(n, hq, d).to(s["q"].dtype), "lse": lse.reshape(n, hq)}


def _plain_delta(s):
    q, k, v, c = s["q"], s["k"], s["v"], _CHUNK
    (t, hk, dk), (h, dv) = q.shape, v.shape[1:]
    off = s["offsets"].long()
    lens = off[1:] - off[:-1]
    n = lens.numel()
    chunks = t // c + n                                                          # (room for every sequence's last, short chunk)
    first = torch.cat([off[:1], torch.cumsum((lens + c - 1) // c, 0)])
    ch = torch.arange(chunks, device=q.device)
    seq = torch.searchsorted(first[1:], ch, right=True)
    real = seq < n
    seq = seq.clamp(max=n - 1)
    i = torch.arange(c, device=q.device)
    tok = off[seq][:, None] + (ch - first[seq])[:, None] * c + i
    on = (tok < off[seq + 1][:, None]) & real[:, None]
    at = tok.clamp(max=t - 1)
    take = lambda x: torch.where(on[:, :, None, None], x[at].float(), 0.0).permute(2, 0, 1, 3)      # noqa: E731  [h, chunk, c, d]
    q, k, v = (take(x).repeat_interleave(h // x.shape[1], 0) for x in (q, k, v))
    fall = torch.cumsum(torch.where(on[:, :, None], s["decay"][at].double(), 0.0), 1).permute(2, 0, 1)      # (64 bits: its differences count)
    beta = torch.where(on[:, :, None], s["beta"][at], 0.0).permute(2, 0, 1)[..., None]
    gap = torch.where(i[:, None] >= i[None, :], torch.exp((fall[..., :, None] - fall[..., None, :]).clamp(max=0)), 0.0).float()
    eye = torch.eye(c, device=q.device)
    low = beta * torch.matmul(k, k.transpose(2, 3)) * gap * (1 - eye)
    # (1 + low)^-1 as a product: low^64 is 0
    inv, power = eye - low, torch.matmul(low, low)
    for _ in range(5):
        inv, power = inv + torch.matmul(inv, power), torch.matmul(power, power)
    scores = torch.matmul(q, k.transpose(2, 3)) * gap
    past, left, whole = torch.exp(fall).float()[..., None], torch.exp(fall[..., -1:] - fall).float()[..., None], torch.exp(fall[..., -1]).float()
    state = torch.zeros(h, n, dk, dv, device=q.device) if s["state"] is None else s["state"].transpose(0, 1)
    o = torch.zeros(h, chunks + 1, c, dv, device=q.device)
    for j in range((s["most"] + c - 1) // c):                                    # the recurrence, a chunk of every sequence at a time
        there = first[:-1] + j < first[1:]
        w = (first[:-1] + j).clamp(max=chunks - 1)
        kw, pw = k[:, w], past[:, w]
        u = torch.matmul(inv[:, w], beta[:, w] * (v[:, w] - pw * torch.matmul(kw, state)))
        o[:, torch.where(there, w, chunks)] = pw * torch.matmul(q[:, w], state) + torch.matmul(scores[:, w], u)
        grown = whole[:, w, None, None] * state + torch.matmul(kw.transpose(2, 3), left[:, w] * u)
        state = torch.where(there[None, :, None, None], grown, state)
    out = torch.empty(t + 1, h, dv, device=q.device)
    out[torch.where(on, tok, t)] = s["sm_scale"] * o[:, :chunks].permute(1, 2, 0, 3)
    return {"out": out[:t].to(s["q"].dtype), "state": state.transpose(0, 1)}


def _plain_delta_step(s):
    h, hk, at = s["v"].shape[1], s["k"].shape[1], s["at"].long()
    q, k = (s[x].float().repeat_interleave(h // hk, 1) for x in "qk")
    state = s["state"][at] * torch.exp(s["decay"])[:, :, None, None]
    u = s["beta"][:, :, None] * (s["v"].float() - (k[..., :, None] * state).sum(-2))
    state = state + k[..., :, None] * u[..., None, :]
    s["state_out"][at] = state
    return {"out": (s["sm_scale"] * (q[..., :, None] * state).sum(-2)).to(s["q"].dtype), "state": s["state_out"]}


def run(state):
    s, op = state, state["op"]
    if not own:
        return {"append_read": _plain_append_read, "read": _plain_read, "attention": _plain_attention, "delta": _plain_delta, "delta_step": _plain_delta_step}[op](s)
    import paper_2506_23906_b200 as mmv

    if op == "append_read":
        mmv.kv_append_q8(s["k"], s["v"], s["offsets"], s["total"], s["table"], *s["cache"], *s["scale"])
        k, v = mmv.kv_read_q8(*s["cache"], *s["scale"], s["all"], s["ends"], s["all"].shape[1] * s["cache"][0].shape[1], dtype=s["k"].dtype)
        return {"k": k, "k_scale": s["scale"][0], "v": v, "v_scale": s["scale"][1]}
    if op == "read":
        k, v = mmv.kv_read_q8(*s["cache"], *s["scale"], s["table"], s["offsets"], s["tokens"], dtype=s["type"])
        return {"k": k, "v": v}
    if op == "attention":
        out, lse = mmv.paged_attention_q8(s["q"], *s["cache"], *s["scale"], s["table"], s["lens"], scale=s["sm_scale"], window=s["window"])
        return {"out": out, "lse": lse}
    if op == "delta":
        out, last = mmv.gated_delta(s["q"], s["k"], s["v"], s["offsets"], s["decay"], s["beta"], scale=s["sm_scale"], state=s["state"])
        return {"out": out, "state": last}
    out = mmv.gated_delta_step(s["q"], s["k"], s["v"], s["decay"], s["beta"], s["state"], scale=s["sm_scale"], slots=s["at"], state_out=s["state_out"])
    return {"out": out, "state": s["state_out"]}


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def _sum_of_lengths(n, most, law, window=0):
    lens = _lengths(random.Random(0), n, most, law)
    return sum(min(x, window) if window else x for x in lens)


def work(case):
    op = case["op"]
    if op == "append_read":     # new values in and out; the blocks that they are in, in and out
        n, most, row = case["nreq"], case["most"], 2 * case["hkv"] * case["d"]
        tokens = n if case["law"] == "decode" else sum(0 if i % 8 == 7 else 1 + i * (most - 1) // max(1, n - 1) for i in range(n))
        held = n * case["block"] if case["law"] == "decode" else tokens + n * case["block"] * 0.6
        return {"bytes": 3.0 * tokens * row + 3 * held * row, "flops": 0}
    if op == "read":
        return {"bytes": 6.0 * _sum_of_lengths(case["nreq"], case["most"], case["law"]) * case["hkv"] * case["d"], "flops": 0}
    if op == "attention":
        tokens = _sum_of_lengths(case["nreq"], case["most"], case["law"], case["window"])
        return {"bytes": 2.0 * tokens * case["hkv"] * (case["d"] + 4.0 / case["block"]) + 4.0 * case["nreq"] * case["hq"] * (case["d"] + 1),
                "flops": 4.0 * tokens * case["hq"] * case["d"]}
    hk, h, dk, dv = case["hk"], case["hk"] * case["rep"], case["dk"], case["dv"]
    if op == "delta":
        t, n = case["tokens"], case["nseq"]
        c = min(_CHUNK, max(1, t // n))
        return {"bytes": 4.0 * t * (hk * dk + h * dv) + 8.0 * t * h + 4.0 * n * h * dk * dv * (2 if case["state"] else 1),
                "flops": 2.0 * t * (c * hk * dk + h * (c * dv + 3 * dk * dv))}
    return {"bytes": case["nreq"] * (h * (8.0 * dk * dv + 4 * dv + 8) + 4.0 * hk * dk), "flops": 7.0 * case["nreq"] * h * dk * dv}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_block(held, old, x, top):
    """One block's new values and scales: held [places, h, d] codes of the scales old [h] (None: a block begun anew), x [tokens, h, d]."""
    amax = x.abs().amax((0, 2))
    if top == 127.0:        # amax / 127, rounded up to 11 significant bits
        unit = torch.exp2(torch.floor(torch.log2((amax / 127).clamp(min=1e-300))) - 10)
        new = torch.ceil(amax / 127 / unit) * unit
    else:
        new = torch.exp2(torch.ceil(torch.log2((amax / 448).clamp(min=1e-300)) - 1e-9))
    new = torch.where(amax < 2.0 ** -100, 0.0, new)
    if old is not None:
        new = torch.where(amax > top * old, new, old)
    per = torch.where(new > 0, new, 1.0)[None, :, None]

    def nearest(y):
        y = y / per
        if top == 127.0:
            return torch.where(y >= 0, torch.floor(y + 0.5), torch.ceil(y - 0.5)) * new[None, :, None]
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)       # of e4m3 around y
        return torch.round(y / step) * step * new[None, :, None]

    kept = None
    if old is not None:
        kept = held.double() * old[None, :, None]
        kept = torch.where((new > old)[None, :, None], nearest(kept), kept)
    return kept, nearest(x), new


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "append_read":     # request by request, block by block
        out = {}
        off, total, table = s["offsets"].tolist(), s["total"].tolist(), s["table"].tolist()
        if off[-1] / s["cache"][0].shape[1] + len(total) > 20000:
            return None
        for name, x, cache, scale in zip("kv", (s["k"], s["v"]), s["cache"], s["scale"]):
            block, top, sc = cache.shape[1], _TOP[cache.dtype], scale.double()
            values = cache.double() * sc[:, None, :, None]
            for r, end in enumerate(total):
                p = end - (off[r + 1] - off[r])
                while p < end:
                    b, lo, hi = table[r][p // block], p % block, min(block, end - p + p % block)
                    new = x[off[r + 1] - (end - p):off[r + 1] - (end - p) + hi - lo].double()
                    kept, written, unit = _exact_block(cache[b, :lo], sc[b] if lo else None, new, top)
                    # what the block's other places hold keeps its codes
                    values[b] = cache[b].double() * unit[None, :, None]
                    if lo:
                        values[b, :lo] = kept
                    values[b, lo:hi] = written
                    sc[b] = unit
                    p += hi - lo
            out[name], out[name + "_scale"] = values.flatten(0, 1), sc
        return out
    if op == "read":
        out = {}
        off = s["offsets"].tolist()
        for name, cache, scale in zip("kv", s["cache"], s["scale"]):
            rows = []
            for r in range(len(off) - 1):
                pages = s["table"][r, : -(-(off[r + 1] - off[r]) // cache.shape[1])].long()
                rows.append((cache[pages].double() * scale[pages].double()[:, None, :, None]).flatten(0, 1)[: off[r + 1] - off[r]])
            out[name] = torch.cat(rows)
        return out
    if op == "attention":       # request by request
        n, hq, d = s["q"].shape
        hkv, block = s["cache"][0].shape[2], s["cache"][0].shape[1]
        out = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
        lse = torch.full((n, hq), -torch.inf, dtype=torch.float64, device="cuda")
        for r, length in enumerate(s["lens"].tolist()):
            if length == 0:
                continue
            pages = s["table"][r, : (length + block - 1) // block].long()
            lo = max(0, length - s["window"]) if s["window"] else 0
            for h in range(hkv):
                k, v = ((c[pages, :, h].double() * w[pages, h].double()[:, None, None]).reshape(-1, d)[lo:length] for c, w in zip(s["cache"], s["scale"]))
                rows = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                x = s["sm_scale"] * (s["q"][r, rows].double() @ k.T)
                lse[r, rows] = torch.logsumexp(x, 1)
                out[r, rows] = torch.softmax(x, 1) @ v
        return {"out": out, "lse": lse}
    h = s["v"].shape[1]
    q, k = (s[x].double().repeat_interleave(h // s[x].shape[1], 1) for x in "qk")
    v, fall, beta = s["v"].double(), torch.exp(s["decay"].double()), s["beta"].double()
    if op == "delta":           # token by token, all sequences and heads side by side
        off = s["offsets"].long()
        lens, n = off[1:] - off[:-1], off.numel() - 1
        (t, _, dk), dv = q.shape, v.shape[2]
        if s["most"] * (1.0 + n * h * dk * dv / 4e6) > 100000:
            return None
        state = torch.zeros(n, h, dk, dv, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
        out = torch.zeros(t + 1, h, dv, dtype=torch.float64, device="cuda")
        for i in range(s["most"]):
            there = i < lens
            tok = torch.where(there, off[:-1] + i, t - 1)
            grown = state * fall[tok][..., None, None]
            u = beta[tok][..., None] * (v[tok] - torch.matmul(k[tok][..., None, :], grown)[..., 0, :])
            grown = grown + k[tok][..., :, None] * u[..., None, :]
            state = torch.where(there[:, None, None, None], grown, state)
            out[torch.where(there, tok, t)] = s["sm_scale"] * torch.matmul(q[tok][..., None, :], grown)[..., 0, :]
        return {"out": out[:t], "state": state}
    at = s["at"].long()
    state = fall[..., None, None] * s["state"][at].double()
    u = beta[..., None] * (v - torch.einsum("nhk,nhkv->nhv", k, state))
    state = state + torch.einsum("nhk,nhv->nhkv", k, u)
    whole = s["state_out"].double()
    whole[at] = state
    return {"out": s["sm_scale"] * torch.einsum("nhk,nhkv->nhv", q, state), "state": whole}
