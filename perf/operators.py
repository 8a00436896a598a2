"""Cases of the operators for serving a language model over a ragged batch: block tables and slot maps, the write into a
paged key-value cache, attention of one new token over that cache, and linear attention with a decay for each head
(packed prompts, single tokens).

``run`` computes a case in its plain form (elementary torch operations in 32 bits) or, with ``own`` set, through the
package's entry points; ``exact`` computes it from the operator's definition in 64 bits.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_CHUNK = 64


# ---------------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decoding step of a busy server: every request grows by a token, few of them into a new block
        {"name": "tables_decode_256", "op": "block_tables", "nreq": 256, "block": 16, "most": 4096, "law": "decode"},
        # a batch of fresh prompts and pieces of prompts, a million new tokens in all
        {"name": "tables_prompts_2048", "op": "block_tables", "nreq": 2048, "block": 32, "most": 1024, "law": "prompts"},
        # the keys and values of one decoding step
        {"name": "append_decode_255", "op": "kv_append", "tokens": 255, "hq": 32, "hkv": 8, "d": 128, "block": 16, "type": "bf16"},
        # a long prompt's
        {"name": "append_prompt_65536", "op": "kv_append", "tokens": 65536, "hq": 16, "hkv": 8, "d": 128, "block": 64, "type": "f16"},
        # a single user's short context: latency
        {"name": "paged_one_777", "op": "paged_attention", "nreq": 1, "hq": 8, "hkv": 2, "d": 64, "block": 16, "most": 777, "law": "same",
         "window": 0, "type": "f16"},
        # an ordinary serving batch, lengths from 0 to 4096, grouped heads
        {"name": "paged_batch_64", "op": "paged_attention", "nreq": 64, "hq": 32, "hkv": 8, "d": 128, "block": 16, "most": 4096, "law": "uniform",
         "window": 0, "type": "bf16"},
        # a few very long contexts: the length has to be split
        {"name": "paged_long_131072", "op": "paged_attention", "nreq": 4, "hq": 32, "hkv": 8, "d": 128, "block": 64, "most": 131072, "law": "same",
         "window": 0, "type": "bf16"},
        # a few short prompts of a small model
        {"name": "linear_prompts_short", "op": "linear_attention", "nseq": 4, "tokens": 333, "h": 4, "dk": 64, "dv": 64, "state": False},
        # an ordinary batch of prompts that continue a state
        {"name": "linear_prompts_batch", "op": "linear_attention", "nseq": 16, "tokens": 32768, "h": 16, "dk": 128, "dv": 128, "state": True},
        # one long prompt: fewer heads than the GPU has processors, so that the length has to be split
        {"name": "linear_prompt_long", "op": "linear_attention", "nseq": 1, "tokens": 65536, "h": 16, "dk": 128, "dv": 128, "state": False},
        # one token of one user
        {"name": "linear_step_1", "op": "linear_step", "nreq": 1, "h": 16, "dk": 128, "dv": 128, "type": "f16"},
        # one token each of a busy server's requests: the states are the traffic
        {"name": "linear_step_256", "op": "linear_step", "nreq": 256, "h": 16, "dk": 128, "dv": 128, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["block_tables", "kv_append", "paged_attention", "paged_attention", "linear_attention", "linear_attention", "linear_step"])
    if op == "block_tables":
        nreq = _log(rng, 1, 4096)
        return {"op": op, "nreq": nreq, "block": rng.choice([8, 16, 32, 48, 64, 128]), "most": _log(rng, 8, max(16, min(8192, 2000000 // nreq))),
                "law": rng.choice(["decode", "prompts"])}
    if op == "kv_append":
        hkv = rng.choice([1, 2, 4, 5, 8])
        return {"op": op, "tokens": _log(rng, 1, 65536), "hq": hkv * rng.choice([1, 2, 4]), "hkv": hkv, "d": rng.choice([64, 80, 96, 128]),
                "block": rng.choice([8, 16, 32, 64, 96]), "type": rng.choice(["bf16", "f16"])}
    if op == "paged_attention":
        hkv, d = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 128, 256])
        nreq = _log(rng, 1, 256)
        most = _log(rng, 16, max(32, min(131072, (1 << 29) // (nreq * hkv * d))))
        return {"op": op, "nreq": nreq, "hq": hkv * rng.choice([1, 2, 4, 6, 8]), "hkv": hkv, "d": d, "block": rng.choice([8, 16, 32, 48, 64, 128]),
                "most": most, "law": rng.choice(["same", "uniform", "skewed"]), "window": rng.choice([0, 0, 0, max(1, most // 3)]),
                "type": rng.choice(["bf16", "f16"])}
    if op == "linear_attention":
        h, dk, dv = rng.choice([1, 2, 4, 6, 8, 16]), rng.choice([64, 96, 128]), rng.choice([64, 80, 128])
        return {"op": op, "nseq": _log(rng, 1, 64), "tokens": _log(rng, 64, 65536), "h": h, "dk": dk, "dv": dv, "state": rng.random() < 0.5}
    return {"op": op, "nreq": _log(rng, 1, 256), "h": rng.choice([1, 4, 6, 12, 16]), "dk": rng.choice([32, 64, 128]), "dv": rng.choice([64, 96, 128]),
            "type": rng.choice(["bf16", "f16"])}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 17)
    return g


def _normal(g, shape, dtype, std=1.0):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    x.normal_(0.0, std, generator=g)
    return x


def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int64)


def _cumulate(x):
    """Exclusive sums of x with the total behind them."""
    return torch.cat([torch.zeros(1, dtype=torch.int64, device=x.device), torch.cumsum(x, 0)])


def _tables(pages, width, ids):
    """A table whose row r holds pages[r] block ids, taken from `ids` in order; 0 behind them."""
    base = _cumulate(pages)
    at = torch.arange(width, device=pages.device)[None, :]
    ids = torch.cat([ids, ids.new_zeros(1)])
    rows = ids[(base[:-1, None] + at).clamp(max=ids.numel() - 1)]
    return torch.where(at < pages[:, None], rows, torch.zeros_like(rows)).to(torch.int32).contiguous()


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    if op == "block_tables":
        n, block, most = case["nreq"], case["block"], case["most"]
        if case["law"] == "decode":
            past, new = _ints(g, 0, most - 1, n), torch.ones(n, dtype=torch.int64, device="cuda")
        else:       # two thirds of the requests are fresh; an eighth of all have nothing to add in this step
            past = torch.where(_ints(g, 0, 2, n) == 0, _ints(g, 0, most, n), 0)
            even = torch.arange(n, device="cuda")       # lengths spread evenly over 1 to most, in any order: every seed fills the batch alike
            new = torch.where(even % 8 == 7, 0, 1 + even * (most - 1) // max(1, n - 1))[torch.randperm(n, generator=g, device="cuda")]
        had = (past + block - 1) // block
        need = (past + new + block - 1) // block
        ids = torch.randperm(int(need.sum()) + 64, generator=g, device="cuda")
        held = int(had.sum())
        tokens = int(new.sum())
        return {"op": op, "block": block, "past": past.to(torch.int32), "new": new.to(torch.int32), "free": ids[held:].to(torch.int32).contiguous(),
                "table": _tables(had, 2 * most // block + 2, ids[:held]), "slots": torch.empty((tokens + 63) // 64 * 64, dtype=torch.int64, device="cuda")}
    if op == "kv_append":
        t, hq, hkv, d, block, dt = case["tokens"], case["hq"], case["hkv"], case["d"], case["block"], _TYPES[case["type"]]
        qkv = _normal(g, (t, hq + 2 * hkv, d), dt)          # the fused projection's output: k and v are views into it
        blocks = (t + block - 1) // block + 3
        ids = torch.randperm(blocks, generator=g, device="cuda")
        at = torch.arange(t, device="cuda")
        slots = torch.where(_ints(g, 0, 31, t) == 0, -1, ids[at // block] * block + at % block)      # -1: padding of the batch
        cache = [torch.zeros(blocks, block, hkv, d, dtype=dt, device="cuda") for _ in range(2)]
        return {"op": op, "k": qkv[:, hq:hq + hkv], "v": qkv[:, hq + hkv:], "slots": slots, "cache": cache}
    if op == "paged_attention":
        n, hq, hkv, d, block, most, dt = (case[x] for x in ("nreq", "hq", "hkv", "d", "block", "most", "type"))
        if case["law"] == "same":
            lens = torch.full((n,), most, dtype=torch.int64, device="cuda")
        elif case["law"] == "uniform":
            lens = _ints(g, 0, most, n)
        else:       # one long context beside many short ones
            lens = _ints(g, 1, max(1, most // 16), n)
            lens[n // 2] = most
        pages = (lens + block - 1) // block
        blocks = int(pages.sum()) + 5
        cache = [_normal(g, (blocks, block, hkv, d), _TYPES[dt]) for _ in range(2)]
        table = _tables(pages, (most + block - 1) // block, torch.randperm(blocks, generator=g, device="cuda"))
        return {"op": op, "q": _normal(g, (n, hq, d), _TYPES[dt]), "cache": cache, "table": table, "lens": lens.to(torch.int32),
                "window": case["window"], "scale": d ** -0.5}
    h, dk, dv = case["h"], case["dk"], case["dv"]
    # decays from fast to slow: a token's weight falls to 1/2 per token in the first head, to 1 - 2^-10 in the last
    decay = torch.log1p(-torch.exp2(-torch.linspace(1, 10, h, device="cuda")))
    if op == "linear_attention":
        t, n = case["tokens"], case["nseq"]
        cuts = torch.sort(_ints(g, 0, t, n - 1))[0] if n > 1 else _ints(g, 0, 0, 0)
        ends = torch.zeros(1, dtype=torch.int64, device="cuda")
        qkv = _normal(g, (t, h, 2 * dk + dv), torch.bfloat16)
        return {"op": op, "q": qkv[..., :dk], "k": qkv[..., dk:2 * dk], "v": qkv[..., 2 * dk:], "decay": decay, "scale": 1.0 / dk,
                "offsets": torch.cat([ends, cuts, ends + t]).to(torch.int32),
                "state": _normal(g, (n, h, dk, dv), torch.float32) if case["state"] else None}
    n, dt = case["nreq"], _TYPES[case["type"]]
    pool = n + n // 4 + 1
    return {"op": op, "q": _normal(g, (n, h, dk), dt), "k": _normal(g, (n, h, dk), dt), "v": _normal(g, (n, h, dv), dt), "decay": decay, "scale": 1.0 / dk,
            "state": _normal(g, (pool, h, dk, dv), torch.float32), "state_out": torch.zeros(pool, h, dk, dv, device="cuda"),
            "at": torch.randperm(pool, generator=g, device="cuda")[:n].to(torch.int32)}


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plain_block_tables(s):
    block, table, free = s["block"], s["table"], s["free"]
    past, new = s["past"].long(), s["new"].long()
    total, off = past + new, _cumulate(new)
    had, need = (past + block - 1) // block, (total + block - 1) // block
    base = _cumulate(need - had)
    at = torch.arange(table.shape[1], device=table.device)[None, :]
    mine = free[(base[:-1, None] + at - had[:, None]).clamp(0, free.numel() - 1)]
    table.copy_(torch.where((at >= had[:, None]) & (at < need[:, None]), mine, table))
    t = torch.arange(s["slots"].numel(), device=table.device)
    r = torch.searchsorted(off[1:], t, right=True).clamp(max=past.numel() - 1)
    p = past[r] + t - off[r]
    slot = table[r, (p // block).clamp(max=table.shape[1] - 1)].long() * block + p % block
    s["slots"].copy_(torch.where(t < off[-1], slot, -1))
    return {"table": table, "slots": s["slots"], "offsets": off.to(torch.int32), "total": total.to(torch.int32), "used": base[-1:].to(torch.int32)}


def _plain_kv_append(s):
    keep = s["slots"] >= 0
    at = s["slots"][keep]
    for cache, x in zip(s["cache"], (s["k"], s["v"])):
        cache.view(-1, *cache.shape[2:])[at] = x[keep]
    return {"k": s["cache"][0], "v": s["cache"][1]}


def _plain_paged_attention(s):
    q, table, lens = s["q"].float(), s["table"].long(), s["lens"].long()
    n, hq, d = q.shape
    kv = [c[table].flatten(1, 2).float() for c in s["cache"]]                    # [request, token, head, d]
    hkv = kv[0].shape[2]
    at = torch.arange(kv[0].shape[1], device=q.device)[None, :]
    on = at < lens[:, None]
    if s["window"]:
        on = on & (at >= lens[:, None] - s["window"])
    x = s["scale"] * torch.einsum("nhgd,nthd->nhgt", q.view(n, hkv, hq // hkv, d), kv[0])
    x = torch.where(on[:, None, None, :], x, -torch.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)                              # (a request of no tokens has only -inf)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = torch.einsum("nhgt,nthd->nhgd", p, kv[1]) / total.clamp(min=1e-38)
    lse = torch.where(total > 0, top + torch.log(total), -torch.inf)
    return {"out": out.reshape(n, hq, d).to(s["q"].dtype), "lse": lse.reshape(n, hq)}


def _plain_linear_attention(s):
    q, k, v, g = s["q"], s["k"], s["v"], s["decay"]
    t, h, dk = q.shape
    dv, off, c = v.shape[2], s["offsets"].long(), _CHUNK
    lens = off[1:] - off[:-1]
    n, chunks = lens.numel(), t // c + lens.numel()                              # (room for every sequence's last, short chunk)
    first = _cumulate((lens + c - 1) // c)
    ch = torch.arange(chunks, device=q.device)
    seq = torch.searchsorted(first[1:], ch, right=True)
    real = seq < n
    seq = seq.clamp(max=n - 1)
    nth = ch - first[seq]                                                        # which chunk of its sequence
    i = torch.arange(c, device=q.device)
    tok = off[seq][:, None] + nth[:, None] * c + i
    on = (tok < off[seq + 1][:, None]) & real[:, None]
    held = on.sum(1)
    take = lambda x: torch.where(on[:, :, None, None], x[tok.clamp(max=t - 1)].float(), 0.0).permute(2, 0, 1, 3)   # noqa: E731  [h, chunk, c, d]
    q, k, v = take(q), take(k), take(v)
    gap = (i[:, None] - i[None, :]).float()
    inside = torch.where(gap >= 0, torch.exp(g[:, None, None] * gap.clamp(min=0)), 0.0)
    o = torch.matmul(torch.matmul(q, k.transpose(2, 3)) * inside[:, None], v)
    left = (held[:, None] - 1 - i[None, :]).clamp(min=0).float()
    kv = torch.matmul((k * torch.exp(g[:, None, None] * left[None])[..., None]).transpose(2, 3), v).reshape(h, chunks, dk * dv)
    # the state in front of every chunk: what the chunks of its sequence before it left, decayed over the chunks between
    lag = nth[:, None] - nth[None, :] - 1
    before = (seq[:, None] == seq[None, :]) & (lag >= 0) & real[:, None] & real[None, :]
    weight = torch.where(before[None], torch.exp(g[:, None, None] * (lag.clamp(min=0) * c).float()[None]), 0.0)
    state = torch.matmul(weight, kv)
    behind = lens[:, None] - (nth * c + held)[None, :]                           # tokens of the sequence behind the chunk
    mine = (torch.arange(n, device=q.device)[:, None] == seq[None, :]) & real[None, :]
    last = torch.matmul(torch.where(mine[None], torch.exp(g[:, None, None] * behind.clamp(min=0).float()[None]), 0.0), kv)
    if s["state"] is not None:
        s0 = s["state"].reshape(n, h, dk * dv).transpose(0, 1)
        state = state + torch.exp(g[:, None] * (nth * c).float()[None])[..., None] * s0[:, seq]
        last = last + torch.exp(g[:, None] * lens.float()[None])[..., None] * s0
    o = o + torch.exp(g[:, None, None] * (i + 1).float())[..., None] * torch.matmul(q, state.view(h, chunks, dk, dv))
    out = torch.empty(t + 1, h, dv, device=q.device)
    out[torch.where(on, tok, t)] = s["scale"] * o.permute(1, 2, 0, 3)
    return {"out": out[:t].to(s["q"].dtype), "state": last.view(h, n, dk, dv).transpose(0, 1)}


def _plain_linear_step(s):
    q, k, v, at = s["q"].float(), s["k"].float(), s["v"].float(), s["at"].long()
    state = s["state"][at] * torch.exp(s["decay"])[:, None, None] + k[..., :, None] * v[..., None, :]
    s["state_out"][at] = state
    return {"out": (s["scale"] * (q[..., :, None] * state).sum(-2)).to(s["q"].dtype), "state": s["state_out"]}


def run(state):
    s, op = state, state["op"]
    if not own:
        return {"block_tables": _plain_block_tables, "kv_append": _plain_kv_append, "paged_attention": _plain_paged_attention,
                "linear_attention": _plain_linear_attention, "linear_step": _plain_linear_step}[op](s)
    import paper_2506_23906_b200 as mmv

    if op == "block_tables":
        off, total, used = mmv.block_tables(s["past"], s["new"], s["free"], s["table"], s["slots"], s["block"])
        return {"table": s["table"], "slots": s["slots"], "offsets": off, "total": total, "used": used}
    if op == "kv_append":
        mmv.kv_append(s["k"], s["v"], s["slots"], s["cache"][0], s["cache"][1])
        return {"k": s["cache"][0], "v": s["cache"][1]}
    if op == "paged_attention":
        out, lse = mmv.paged_attention(s["q"], s["cache"][0], s["cache"][1], s["table"], s["lens"], scale=s["scale"], window=s["window"])
        return {"out": out, "lse": lse}
    if op == "linear_attention":
        out, last = mmv.linear_attention(s["q"], s["k"], s["v"], s["offsets"], s["decay"], scale=s["scale"], state=s["state"])
        return {"out": out, "state": last}
    out = mmv.linear_attention_step(s["q"], s["k"], s["v"], s["decay"], s["state"], scale=s["scale"], slots=s["at"], state_out=s["state_out"])
    return {"out": out, "state": s["state_out"]}


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "block_tables":
        n, block, most = case["nreq"], case["block"], case["most"]
        tokens = n if case["law"] == "decode" else n * 7 / 8 * (most + 1) / 2
        fresh = tokens / block
        # lengths in, offsets and totals out, a slot per token, an id per new block in and out
        return {"bytes": 16.0 * n + 8 * tokens + 8 * fresh, "flops": 0}
    if op == "kv_append":
        return {"bytes": case["tokens"] * (31 / 32 * 8 * case["hkv"] * case["d"] + 8.0), "flops": 0}
    if op == "paged_attention":
        n, most, win = case["nreq"], case["most"], case["window"] or case["most"]
        short = max(1, most // 16)
        mean = lambda top: top / 2 if win >= top else win - win * win / (2.0 * top)   # noqa: E731  of min(length, window), length uniform up to top
        tokens = n * min(most, win) if case["law"] == "same" else n * mean(most) if case["law"] == "uniform" else min(most, win) + (n - 1) * mean(short)
        return {"bytes": 4.0 * tokens * case["hkv"] * case["d"] + 4.0 * n * case["hq"] * (case["d"] + 1), "flops": 4.0 * tokens * case["hq"] * case["d"]}
    h, dk, dv = case["h"], case["dk"], case["dv"]
    if op == "linear_attention":
        t, n = case["tokens"], case["nseq"]
        c = min(_CHUNK, max(1, t // n))
        return {"bytes": 4.0 * t * h * (dk + dv) + 4.0 * n * h * dk * dv * (2 if case["state"] else 1),
                "flops": 2.0 * t * h * (c / 2 * (dk + dv) + 2 * dk * dv)}
    return {"bytes": case["nreq"] * h * (8.0 * dk * dv + 4 * (dk + dv)), "flops": 5.0 * case["nreq"] * h * dk * dv}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "block_tables":        # whole numbers: request by request on the host
        past, new, free, table, block = s["past"].tolist(), s["new"].tolist(), s["free"].tolist(), s["table"].tolist(), s["block"]
        slots, off, used = [], [0], 0
        for r in range(len(past)):
            for p in range(past[r], past[r] + new[r]):
                if p % block == 0:
                    table[r][p // block] = free[used]
                    used += 1
                slots.append(table[r][p // block] * block + p % block)
            off.append(len(slots))
        slots += [-1] * (s["slots"].numel() - len(slots))
        i32 = torch.int32
        return {"table": torch.tensor(table, dtype=i32), "slots": torch.tensor(slots), "offsets": torch.tensor(off, dtype=i32),
                "total": torch.tensor([a + b for a, b in zip(past, new)], dtype=i32), "used": torch.tensor([used], dtype=i32)}
    if op == "kv_append":
        out = [c.double() for c in s["cache"]]
        block = out[0].shape[1]
        there = torch.nonzero(s["slots"] >= 0)[:, 0]
        for c, x in zip(out, (s["k"], s["v"])):
            c[s["slots"][there] // block, s["slots"][there] % block] = x[there].double()
        return {"k": out[0], "v": out[1]}
    if op == "paged_attention":     # request by request
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
                k, v = (c[pages, :, h].reshape(-1, d)[lo:length].double() for c in s["cache"])
                rows = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                x = s["scale"] * (s["q"][r, rows].double() @ k.T)
                lse[r, rows] = torch.logsumexp(x, 1)
                out[r, rows] = torch.softmax(x, 1) @ v
        return {"out": out, "lse": lse}
    if op == "linear_attention":    # token by token, all sequences and heads side by side
        q, k, v, off = s["q"].double(), s["k"].double(), s["v"].double(), s["offsets"].long()
        lens, n = off[1:] - off[:-1], s["offsets"].numel() - 1
        t, h, dk = q.shape
        dv, fall = v.shape[2], torch.exp(s["decay"].double())[None, :, None, None]
        if int(lens.max()) * (1.0 + n * h * dk * dv / 4e6) > 150000:
            return None
        state = torch.zeros(n, h, dk, dv, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
        out = torch.zeros(t + 1, h, dv, dtype=torch.float64, device="cuda")
        for i in range(int(lens.max())):
            there = i < lens
            tok = torch.where(there, off[:-1] + i, t - 1)
            grown = state * fall + k[tok][..., :, None] * v[tok][..., None, :]
            state = torch.where(there[:, None, None, None], grown, state)
            out[torch.where(there, tok, t)] = s["scale"] * torch.matmul(q[tok][..., None, :], grown)[..., 0, :]
        return {"out": out[:t], "state": state}
    at = s["at"].long()
    state = torch.exp(s["decay"].double())[:, None, None] * s["state"][at].double()
    state += torch.einsum("nhk,nhv->nhkv", s["k"].double(), s["v"].double())
    whole = s["state_out"].double()
    whole[at] = state
    return {"out": s["scale"] * torch.einsum("nhk,nhkv->nhv", s["q"].double(), state), "state": whole}
