"""A two-layer decoder served over a ragged batch with the library's operators: prompts, then single tokens.

    python examples/serve_ragged_batch.py [--requests 6] [--steps 8] [--check]

One layer keeps a decayed state (linear attention), the other a paged key-value cache (softmax attention).  A step of the server
is always the same five calls: block_tables (offsets, slots, new table entries), then per layer its projection and
linear_attention or linear_attention_step, kv_append and paged_attention.  Weights are random.  --check recomputes the last
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


class Server:
    def __init__(self, requests: int, longest: int, seed: int = 0):
        g = torch.Generator("cuda").manual_seed(seed)
        w = lambda *s: (torch.randn(*s, device="cuda", generator=g) * s[0] ** -0.5).bfloat16()      # noqa: E731
        self.embed, self.head = w(VOCAB, WIDTH) * VOCAB ** 0.5, w(WIDTH, VOCAB)
        self.lin_in, self.lin_out = w(WIDTH, 3 * HEADS * DIM), w(HEADS * DIM, WIDTH)
        self.att_in, self.att_out = w(WIDTH, (HEADS + 2 * KV_HEADS) * DIM), w(HEADS * DIM, WIDTH)
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(2, 8, HEADS, device="cuda")))
        # what a server keeps: the pool of blocks, the requests' tables and lengths, the layers' states
        blocks = requests * (-(-longest // BLOCK)) + 2
        self.cache = [torch.empty(blocks, BLOCK, KV_HEADS, DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.free = torch.randperm(blocks, device="cuda", generator=g).to(torch.int32)
        self.table = torch.zeros(requests, -(-longest // BLOCK), dtype=torch.int32, device="cuda")
        self.past = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.state = torch.zeros(requests, HEADS, DIM, DIM, device="cuda")

    def step(self, tokens: torch.Tensor, counts: list[int]) -> torch.Tensor:
        """tokens: the batch's new tokens, packed; counts: how many of each request.  Returns every token's logits."""
        n, requests = tokens.numel(), len(counts)
        added = torch.tensor(counts, dtype=torch.int32, device="cuda")
        slots = torch.empty(n, dtype=torch.int64, device="cuda")
        offsets, total, used = mmv.block_tables(self.past, added, self.free, self.table, slots, BLOCK)
        x = self.embed[tokens]
        single = all(c == 1 for c in counts)                            # a decoding step: one token of every request

        q, k, v = (norm(x) @ self.lin_in).view(n, 3, HEADS, DIM).unbind(1)
        if single:
            o = mmv.linear_attention_step(q, k, v, self.log_decay, self.state, scale=DIM ** -0.5)
        else:
            o, self.state = mmv.linear_attention(q, k, v, offsets, self.log_decay, scale=DIM ** -0.5, state=self.state)
        x = x + norm(o.reshape(n, -1)) @ self.lin_out

        qkv = (norm(x) @ self.att_in).view(n, HEADS + 2 * KV_HEADS, DIM)
        mmv.kv_append(qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:], slots, *self.cache)
        if single:
            o, _ = mmv.paged_attention(qkv[:, :HEADS], *self.cache, self.table, total)
        else:       # every token of a prompt attends to those in front of it: a request of its own over the same pages
            owner = torch.repeat_interleave(torch.arange(requests, device="cuda"), added.long(), output_size=n)
            seen = (self.past[owner] + torch.arange(1, n + 1, device="cuda") - offsets[owner]).to(torch.int32)
            o, _ = mmv.paged_attention(qkv[:, :HEADS], *self.cache, self.table[owner], seen)
        x = x + o.reshape(n, -1) @ self.att_out

        self.past = total
        self.free = self.free[int(used):]                               # (the scheduler's book-keeping, on the host)
        return (norm(x) @ self.head).float()

    def dense(self, tokens: torch.Tensor, rounded: bool = False) -> torch.Tensor:
        """The same model over one whole sequence, in fp32 and without a cache: the last token's logits.  rounded: with activations
        rounded to bfloat16 where the server's are, which says how much of a difference the model makes of that rounding."""
        f = lambda w: w.float()                                         # noqa: E731
        r = (lambda x: x.bfloat16().float()) if rounded else (lambda x: x)
        n = tokens.numel()
        x = f(self.embed)[tokens]
        q, k, v = r(r(norm(x)) @ f(self.lin_in)).view(n, 3, HEADS, DIM).permute(1, 2, 0, 3)
        i = torch.arange(n, device="cuda")
        gap = (i[:, None] - i[None, :]).float()
        fall = torch.where(gap >= 0, torch.exp(self.log_decay[:, None, None] * gap.clamp(min=0)), 0.0)
        o = r(((q @ k.transpose(1, 2) * fall) @ v * DIM ** -0.5).transpose(0, 1).reshape(n, -1))
        x = r(x + r(r(norm(o)) @ f(self.lin_out)))
        qkv = r(r(norm(x)) @ f(self.att_in)).view(n, -1, DIM).transpose(0, 1)
        rep = HEADS // KV_HEADS
        q, k, v = qkv[:HEADS], qkv[HEADS:HEADS + KV_HEADS].repeat_interleave(rep, 0), qkv[HEADS + KV_HEADS:].repeat_interleave(rep, 0)
        p = torch.softmax(torch.where(gap >= 0, q @ k.transpose(1, 2) * DIM ** -0.5, -torch.inf), -1)
        x = r(x + r(r((p @ v).transpose(0, 1).reshape(n, -1)) @ f(self.att_out)))
        return r(r(norm(x[-1:]))[0] @ f(self.head))


def serve(requests: int, steps: int, seed: int = 0):
    """Prompts of ragged lengths and `steps` greedy tokens each.  Returns (server, token sequences, the last step's logits)."""
    g = torch.Generator().manual_seed(seed)
    lens = (torch.randint(1, 200, (requests,), generator=g)).tolist()
    texts = [torch.randint(0, VOCAB, (n,), generator=g).cuda() for n in lens]
    server = Server(requests, max(lens) + steps + 1, seed)
    logits = server.step(torch.cat(texts), lens)
    last = logits[torch.tensor(lens).cumsum(0) - 1]
    for _ in range(steps):
        token = last.argmax(-1)
        texts = [torch.cat([t, token[r:r + 1]]) for r, t in enumerate(texts)]
        last = server.step(token, [1] * requests)
    return server, texts, last


def serve_in_pieces(schedule: list[list[int]], seed: int = 0):
    """Random tokens, schedule[i][r] of them from request r in step i (none of some is fine).  Returns what serve() does, every request's
    logits from the last step that it had a token in."""
    g = torch.Generator().manual_seed(seed)
    requests = len(schedule[0])
    server = Server(requests, sum(map(max, schedule)) + 1, seed)
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
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    server, texts, last = serve(a.requests, a.steps)
    for r, t in enumerate(texts):
        print(f"request {r}: {t.numel()} tokens, the last ones {t[-min(a.steps, 8):].tolist()}")
    fine = True
    if a.check:
        for name, run in (("prompts and single tokens", (server, texts, last)), ("pieces", serve_in_pieces(PIECES))):
            off, own = difference(*run)
            print(f"{name}: last logits against the dense fp32 model: relative difference {off:.2e}; of the dense model with rounded activations: {own:.2e}")
            fine &= off < 2 * own
    return 0 if fine else 1


if __name__ == "__main__":
    sys.exit(main())
