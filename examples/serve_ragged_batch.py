"""A two-layer decoder served over a ragged batch with the library's operators: prompts, then single tokens.

    python examples/serve_ragged_batch.py [--requests 6] [--steps 8] [--cache bf16|int8|e4m3] [--delta] [--check]

One layer keeps a decayed state (linear attention), the other a paged key-value cache (softmax attention).  A step of the server
is always the same five calls: block_tables (offsets, slots, new table entries), then per layer its projection and
linear_attention or linear_attention_step, kv_append and paged_attention.  With --cache int8 or e4m3 the cache is held in 8 bits
(kv_append_q8; single tokens attend with paged_attention_q8, prompts to what kv_read_q8 brings back of their requests), with --delta the
state follows the gated delta rule (gated_delta, gated_delta_step).  Weights are random.  --check recomputes the last
step's logits from the whole token sequences with dense fp32 attention, for that run and for one whose requests add none, one or two
tokens in a step.
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
import paper_2506_23906_b200 as mmv  # noqa: E402

VOCAB, WIDTH, HEADS, KV_HEADS, DIM, BLOCK = 512, 512, 8, 2, 64, 16
PIECES = [[40, 0, 17], [1, 1, 1], [2, 0, 1], [0, 3, 0], [0, 1, 2], [1, 2, 0], [1, 1, 1]]       # --check: tokens of each request in each step


def norm(x: torch.Tensor) -> torch.Tensor:
    """Every row divided by its root mean square, in fp32."""
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def unit(x: torch.Tensor) -> torch.Tensor:
    """Every row divided by its length, in fp32."""
    y = x.float()
    return (y * torch.rsqrt(y.square().sum(-1, keepdim=True) + 1e-6)).to(x.dtype)


def in_8_bits(x: torch.Tensor, code: torch.dtype) -> torch.Tensor:
    """[tokens, heads, dim] as a cache in 8 bits gives them back: blocks of BLOCK tokens, a scale for each and head."""
    n, top = x.size(0), 127.0 if code == torch.int8 else 448.0
    y = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, -n % BLOCK)).view(-1, BLOCK, *x.shape[1:])
    m, e = torch.frexp(y.abs().amax((1, 3), keepdim=True).clamp(min=1e-30) / top)
    scale = torch.ldexp(torch.ceil(m * 2048) / 2048 if code == torch.int8 else torch.ones_like(m), e)
    codes = torch.round(y / scale) if code == torch.int8 else (y / scale).to(code).float()
    return (codes * scale).flatten(0, 1)[:n]


class Server:
    def __init__(self, requests: int, longest: int, seed: int = 0, cache: str = "bf16", delta: bool = False):
        g = torch.Generator("cuda").manual_seed(seed)
        w = lambda *s: (torch.randn(*s, device="cuda", generator=g) * s[0] ** -0.5).bfloat16()      # noqa: E731
        self.embed, self.head = w(VOCAB, WIDTH) * VOCAB ** 0.5, w(WIDTH, VOCAB)
        self.lin_in, self.lin_out = w(WIDTH, 3 * HEADS * DIM), w(HEADS * DIM, WIDTH)
        self.att_in, self.att_out = w(WIDTH, (HEADS + 2 * KV_HEADS) * DIM), w(HEADS * DIM, WIDTH)
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(2, 8, HEADS, device="cuda")))
        # what a server keeps: the pool of blocks, the requests' tables and lengths, the layers' states
        blocks = requests * (-(-longest // BLOCK)) + 2
        self.code = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[cache]
        self.cache = [torch.empty(blocks, BLOCK, KV_HEADS, DIM, dtype=self.code, device="cuda") for _ in range(2)]
        self.free = torch.randperm(blocks, device="cuda", generator=g).to(torch.int32)
        self.table = torch.zeros(requests, -(-longest // BLOCK), dtype=torch.int32, device="cuda")
        self.past = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.state = torch.zeros(requests, HEADS, DIM, DIM, device="cuda")
        if cache != "bf16":                                             # scales of the codes, one for each block and head
            self.cache += [torch.zeros(blocks, KV_HEADS, device="cuda") for _ in range(2)]
        self.delta = delta
        if delta:                                                       # every token's decay and beta
            self.gates = w(WIDTH, 2 * HEADS)

    def step(self, tokens: torch.Tensor, counts: list[int]) -> torch.Tensor:
        """tokens: the batch's new tokens, packed; counts: how many of each request.  Returns every token's logits."""
        n, requests = tokens.numel(), len(counts)
        added = torch.tensor(counts, dtype=torch.int32, device="cuda")
        slots = torch.empty(n, dtype=torch.int64, device="cuda")
        offsets, total, used = mmv.block_tables(self.past, added, self.free, self.table, slots, BLOCK)
        x = self.embed[tokens]
        single = all(c == 1 for c in counts)                            # a decoding step: one token of every request

        q, k, v = (norm(x) @ self.lin_in).view(n, 3, HEADS, DIM).unbind(1)
        if self.delta:
            q, k, (decay, beta) = unit(q), unit(k), self.gated(norm(x) @ self.gates)
            if single:
                o = mmv.gated_delta_step(q, k, v, decay, beta, self.state)
            else:
                o, _ = mmv.gated_delta(q, k, v, offsets, decay, beta, state=self.state, state_out=self.state)
        elif single:
            o = mmv.linear_attention_step(q, k, v, self.log_decay, self.state, scale=DIM ** -0.5)
        else:
            o, self.state = mmv.linear_attention(q, k, v, offsets, self.log_decay, scale=DIM ** -0.5, state=self.state)
        x = x + norm(o.reshape(n, -1)) @ self.lin_out

        qkv = (norm(x) @ self.att_in).view(n, HEADS + 2 * KV_HEADS, DIM)
        new = qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]
        if self.code == torch.bfloat16:
            mmv.kv_append(*new, slots, *self.cache)
            attend = mmv.paged_attention
        else:
            mmv.kv_append_q8(*new, offsets, total, self.table, *self.cache)
            attend = mmv.paged_attention_q8
        if single:
            o, _ = attend(qkv[:, :HEADS], *self.cache, self.table, total)
        else:       # every token of a prompt attends to those in front of it
            owner = torch.repeat_interleave(torch.arange(requests, device="cuda"), added.long(), output_size=n)
            seen = (self.past[owner] + torch.arange(1, n + 1, device="cuda") - offsets[owner]).to(torch.int32)
            if self.code == torch.bfloat16:                             # as a request of its own over the same pages
                o, _ = mmv.paged_attention(qkv[:, :HEADS], *self.cache, self.table[owner], seen)
            else:                                                       # in what its request holds, back in 16 bits
                o = self.prompt_attention(qkv[:, :HEADS], total, owner, seen)
        x = x + o.reshape(n, -1) @ self.att_out

        self.past = total
        self.free = self.free[int(used):]                               # (the scheduler's book-keeping, on the host)
        return (norm(x) @ self.head).float()

    def gated(self, x: torch.Tensor):
        """Decay (its logarithm) and beta of every token and head from the gates' projection."""
        x = x.float().view(-1, 2, HEADS)
        return -torch.nn.functional.softplus(x[:, 0]) * torch.exp(self.log_decay).neg().add(1), torch.sigmoid(x[:, 1])

    def prompt_attention(self, q: torch.Tensor, total: torch.Tensor, owner: torch.Tensor, seen: torch.Tensor) -> torch.Tensor:
        """Attention of several new tokens per request, over their requests' whole contents read back from the 8-bit cache."""
        ends = torch.cat([torch.zeros_like(total[:1]), total.cumsum(0, dtype=torch.int32)])
        held = int(ends[-1])
        k, v = mmv.kv_read_q8(*self.cache, self.table, ends, held)
        of = torch.repeat_interleave(torch.arange(total.numel(), device="cuda"), total.long(), output_size=held)
        place = torch.arange(held, device="cuda") - ends[of]
        on = (of[None, :] == owner[:, None]) & (place[None, :] < seen[:, None])
        rep = HEADS // KV_HEADS
        x = torch.einsum("nhd,mhd->hnm", q.float(), k.float().repeat_interleave(rep, 1)) * DIM ** -0.5
        p = torch.softmax(torch.where(on, x, -torch.inf), -1)
        return torch.einsum("hnm,mhd->nhd", p, v.float().repeat_interleave(rep, 1)).to(q.dtype)

    def dense(self, tokens: torch.Tensor, rounded: bool = False) -> torch.Tensor:
        """The same model over one whole sequence, in fp32 and without a cache: the last token's logits.  rounded: with activations
        rounded to bfloat16 where the server's are (and keys and values to 8 bits, if its cache holds them so), which says how much of a
        difference the model makes of that rounding."""
        f = lambda w: w.float()                                         # noqa: E731
        r = (lambda x: x.bfloat16().float()) if rounded else (lambda x: x)
        n = tokens.numel()
        x = f(self.embed)[tokens]
        q, k, v = r(r(norm(x)) @ f(self.lin_in)).view(n, 3, HEADS, DIM).permute(1, 2, 0, 3)
        i = torch.arange(n, device="cuda")
        gap = (i[:, None] - i[None, :]).float()
        fall = torch.where(gap >= 0, torch.exp(self.log_decay[:, None, None] * gap.clamp(min=0)), 0.0)
        if self.delta:
            decay, beta = self.gated(r(r(norm(x)) @ f(self.gates)))
            q, k, state, o = r(unit(q)), r(unit(k)), torch.zeros(HEADS, DIM, DIM, device="cuda"), torch.empty(n, HEADS, DIM, device="cuda")
            for t in range(n):
                state = torch.exp(decay[t])[:, None, None] * state
                u = beta[t][:, None] * (v[:, t] - (k[:, t, None, :] @ state)[:, 0])
                state = state + k[:, t, :, None] * u[:, None, :]
                o[t] = (q[:, t, None, :] @ state)[:, 0]
            o = r(o.reshape(n, -1))
        else:
            o = r(((q @ k.transpose(1, 2) * fall) @ v * DIM ** -0.5).transpose(0, 1).reshape(n, -1))
        x = r(x + r(r(norm(o)) @ f(self.lin_out)))
        qkv = r(r(norm(x)) @ f(self.att_in)).view(n, -1, DIM).transpose(0, 1)
        if rounded and self.code != torch.bfloat16:
            qkv = torch.cat([qkv[:HEADS], in_8_bits(qkv[HEADS:].transpose(0, 1), self.code).transpose(0, 1)])
        rep = HEADS // KV_HEADS
        q, k, v = qkv[:HEADS], qkv[HEADS:HEADS + KV_HEADS].repeat_interleave(rep, 0), qkv[HEADS + KV_HEADS:].repeat_interleave(rep, 0)
        p = torch.softmax(torch.where(gap >= 0, q @ k.transpose(1, 2) * DIM ** -0.5, -torch.inf), -1)
        x = r(x + r(r((p @ v).transpose(0, 1).reshape(n, -1)) @ f(self.att_out)))
        return r(r(norm(x[-1:]))[0] @ f(self.head))


def serve(requests: int, steps: int, seed: int = 0, **how):
    """Prompts of ragged lengths and `steps` greedy tokens each.  Returns (server, token sequences, the last step's logits)."""
    g = torch.Generator().manual_seed(seed)
    lens = (torch.randint(1, 200, (requests,), generator=g)).tolist()
    texts = [torch.randint(0, VOCAB, (n,), generator=g).cuda() for n in lens]
    server = Server(requests, max(lens) + steps + 1, seed, **how)
    logits = server.step(torch.cat(texts), lens)
    last = logits[torch.tensor(lens).cumsum(0) - 1]
    for _ in range(steps):
        token = last.argmax(-1)
        texts = [torch.cat([t, token[r:r + 1]]) for r, t in enumerate(texts)]
        last = server.step(token, [1] * requests)
    return server, texts, last


def serve_in_pieces(schedule: list[list[int]], seed: int = 0, **how):
    """Random tokens, schedule[i][r] of them from request r in step i (none of some is fine).  Returns what serve() does, every request's
    logits from the last step that it had a token in."""
    g = torch.Generator().manual_seed(seed)
    requests = len(schedule[0])
    server = Server(requests, sum(map(max, schedule)) + 1, seed, **how)
    texts, last = [torch.empty(0, dtype=torch.int64, device="cuda")] * requests, torch.zeros(requests, VOCAB, device="cuda")
    for counts in schedule:
        new = [torch.randint(0, VOCAB, (c,), generator=g).cuda() for c in counts]
        texts = [torch.cat(t) for t in zip(texts, new)]
        logits = server.step(torch.cat(new), counts)
        ends = torch.tensor(counts).cumsum(0) - 1
        for r, c in enumerate(counts):
            if c:
                last[r] = logits[ends[r]]
    return server, texts, last


def difference(server: Server, texts, last: torch.Tensor):
    """How far the served logits, and those of the dense model with rounded activations, are from the dense fp32 model's."""
    want, rounded = (torch.stack([server.dense(t, r) for t in texts]) for r in (False, True))
    return float((last - want).norm() / want.norm()), float((rounded - want).norm() / want.norm())


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=6)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--cache", choices=["bf16", "int8", "e4m3"], default="bf16")
    ap.add_argument("--delta", action="store_true")
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    how = {"cache": a.cache, "delta": a.delta}
    server, texts, last = serve(a.requests, a.steps, **how)
    for r, t in enumerate(texts):
        print(f"request {r}: {t.numel()} tokens, the last ones {t[-min(a.steps, 8):].tolist()}")
    fine = True
    if a.check:
        for name, run in (("prompts and single tokens", (server, texts, last)), ("pieces", serve_in_pieces(PIECES, **how))):
            off, own = difference(*run)
            print(f"{name}: last logits against the dense fp32 model: relative difference {off:.2e}; of the dense model with rounded activations: {own:.2e}")
            fine &= off < 2 * own
    return 0 if fine else 1


if __name__ == "__main__":
    sys.exit(main())
