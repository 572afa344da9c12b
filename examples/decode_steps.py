#!/usr/bin/env python3
"""Decode steps of a small mixture-of-experts model over a paged cache.

A batch of requests of different lengths is served to its end: in every step each request's place for one more token
is found on the GPU (KvTables), and in every layer the token's key and value rows are written (KvCache.append), its
attention over the request's cached tokens is computed (DecodeAttention), and its experts under the layer's plan
(RankForward, one rank).  Projections are torch's.  Requests end on the way, their pages go back, and a waiting request
takes over the free row.  A step in which no request arrives always launches the same work, so it is recorded once and
replayed; the step's tokens per request are its only input.

    python examples/decode_steps.py [--cache bf16|e4m3|latent|latent_e4m3] [--steps N] [--page-size P] [--eager]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import numpy as np
import torch

from paper_2603_28768_amd import binding, synth

CONFIG = synth.scaled(synth.CONFIGS["qwen3"], H=256, I=128, E=16, k=4, D=1, replica_slots=0)
LAYERS, VOCABULARY, HEADS = 2, 512, 8


def cache_rows(cache):
    """Heads of a layer's cache, elements of a key row and of a value row.  Latent rows, which all query heads share, are
    as long as models have them: those of up to 256 elements go through the kernel of ordinary rows."""
    return (1, 576, 512) if cache.startswith("latent") else (HEADS // 4, 64, 64)


class Layer:
    """Weights, cache and kernels of one layer; `hidden` is the step's activations, one row per request."""

    def __init__(self, plan, index, R, pages, page_size, max_pages, cache, gen, device):
        H = CONFIG.H
        matrix = lambda rows, cols: (torch.randn((cols, rows), generator=gen, device=device) * rows ** -0.5).bfloat16()  # noqa: E731
        latent = cache.startswith("latent")
        self.heads, self.dk, self.dv = cache_rows(cache)
        self.cache = binding.KvCache.allocate(pages, page_size, self.heads, self.dk, self.dv, "e4m3" if cache.endswith("e4m3") else "bf16",
                                              latent=latent, device=device)
        self.attention = binding.DecodeAttention(self.cache, R, HEADS, max_pages)
        self.w_q, self.w_k, self.w_out = matrix(H, HEADS * self.dk), matrix(H, self.heads * self.dk), matrix(HEADS * self.dv, H)
        self.w_v = None if latent else matrix(H, self.heads * self.dv)
        experts = [[binding.to_device(m, "bf16", device) for m in synth.expert_weights(CONFIG, e, index)] for e in range(CONFIG.E)]
        self.experts = binding.RankForward(plan, index, 0, "bf16", R, H, CONFIG.I, CONFIG.k, *zip(*experts), packed=[binding.pack_weights(*w) for w in experts],
                                           w_router=binding.to_device(synth.gate_weights(CONFIG, index), "bf16", device), device=device)

    def append(self, hidden, slots):
        rows = lambda w, d: None if w is None else (hidden @ w.T).view(-1, self.heads, d)  # noqa: E731
        self.cache.append(rows(self.w_k, self.dk), rows(self.w_v, self.dv), slots)

    def step(self, hidden, slots, tables):
        x = norm(hidden)
        self.append(x, slots)
        self.q = (x @ self.w_q.T).view(-1, HEADS, self.dk)
        attended = self.attention(self.q, tables.lens, tables.table)
        hidden = hidden + attended.reshape(len(hidden), -1) @ self.w_out.T
        return hidden + self.experts(norm(hidden))


def norm(x):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(dim=1, keepdim=True) + 1e-6)).bfloat16()


class Server:
    def __init__(self, R: int, longest: int, page_size: int = 16, cache: str = "bf16", seed: int = 0, device="cuda:0"):
        gen = torch.Generator(device=device).manual_seed(seed)
        max_pages = -(-longest // page_size)
        pages = R * max_pages
        loads = np.ones((1, LAYERS, CONFIG.E), dtype=np.int64)
        plan = binding.Plan(loads, CONFIG.D, CONFIG.replica_slots)
        self.R, self.longest = R, longest
        table = lambda rows, size: (torch.randn((rows, CONFIG.H), generator=gen, device=device) * size).bfloat16()  # noqa: E731
        self.embedding, self.place, self.head = table(VOCABULARY, 0.3), table(longest, 0.1), table(VOCABULARY, 1.0)
        self.layers = [Layer(plan, i, R, pages, page_size, max_pages, cache, gen, device) for i in range(LAYERS)]
        self.tables = binding.KvTables(R, max_pages, pages, page_size, R, device=device)
        # the same state with room for a prompt's tokens in a step
        t = self.tables
        self.prompt_tables = binding.KvTables(R, max_pages, pages, page_size, longest, lens=t.lens, table=t.table, ring=t.ring, pool=t.pool)
        self.add = torch.zeros(R, dtype=torch.int32, device=device)
        self.token = torch.zeros(R, dtype=torch.int64, device=device)
        self.graph = None

    def arrive(self, row: int, prompt):
        """A request takes over an empty row: its prompt's rows go into every layer's cache, here from the
        embeddings alone (another instance's prefill in earnest), its last token is answered by the next step."""
        add = torch.zeros_like(self.add)
        add[row] = len(prompt) - 1
        slots = self.prompt_tables.step(add)
        ids = torch.zeros(self.longest, dtype=torch.int64, device=add.device)
        ids[:len(prompt) - 1] = prompt[:-1]
        hidden = norm(self.embedding[ids] + self.place[self.prompt_tables.positions.long().clamp(min=0)])
        for layer in self.layers:
            layer.append(hidden, slots)                       # slots behind the prompt's are -1: nothing is written
        self.token[row] = prompt[-1]

    def decode(self):
        """One step of all rows: self.add has 1 where a request goes on, -1 where it has ended, 0 for empty rows."""
        t = self.tables
        slots = t.step(self.add)
        # requests without a token have none among `slots`: one slot per row, -1 where there is nothing to write
        slot = torch.where(self.add > 0, slots[t.token_off[:-1].long().clamp(max=self.R - 1)], -1)
        hidden = self.embedding[self.token] + self.place[(t.lens - 1).long().clamp(min=0)]
        for layer in self.layers:
            hidden = layer.step(hidden, slot, t)
        logits = norm(hidden).float() @ self.head.float().T
        self.token.copy_(torch.where(self.add > 0, logits.argmax(dim=1), self.token))

    def record(self):
        """Record a step; with all rows at 0, recording and its warm-up change no state."""
        self.add.zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.decode()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.decode()

    def step(self, add):
        self.add.copy_(add)
        if self.graph is None:
            self.decode()
        else:
            self.graph.replay()


def serve(R=8, steps=24, page_size=16, cache="bf16", eager=False, seed=0, longest=256, device="cuda:0"):
    """Serves requests of seeded prompts and lengths for so many steps.  Returns the server and the answered tokens of every
    request, in the order of arrival."""
    rng = np.random.default_rng(seed)
    server = Server(R, longest, page_size, cache, seed, device)
    if not eager:
        server.record()
    answers, left, who = [], [0] * R, [None] * R
    for _ in range(steps):
        ending = [who[r] is not None and left[r] == 0 for r in range(R)]
        if any(ending):                                       # pages go back before new requests ask for some
            server.step(torch.tensor([-1 if e else 0 for e in ending], dtype=torch.int32))
        for r in range(R):
            if who[r] is None or ending[r]:
                prompt = torch.from_numpy(rng.integers(0, VOCABULARY, int(rng.integers(1, longest // 2)))).to(device)
                server.arrive(r, prompt)
                who[r], left[r] = len(answers), int(rng.integers(1, longest // 4))
                answers.append([])
        server.step(torch.ones(R, dtype=torch.int32))
        tokens = server.token.tolist()
        for r in range(R):
            answers[who[r]].append(tokens[r])
            left[r] -= 1
    return server, answers


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cache", choices=["bf16", "e4m3", "latent", "latent_e4m3"], default="bf16")
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--page-size", type=int, default=16)
    ap.add_argument("--eager", action="store_true", help="launch every step anew instead of replaying a recorded one")
    a = ap.parse_args()
    torch.zeros(1, device="cuda:0")
    t0 = time.perf_counter()
    server, answers = serve(a.requests, a.steps, a.page_size, a.cache, a.eager)
    torch.cuda.synchronize()
    print(f"{len(answers)} requests, {sum(map(len, answers))} tokens in {time.perf_counter() - t0:.2f} s; cached tokens now {server.tables.lens.tolist()}, "
          f"free pages {int(server.tables.pool[1] - server.tables.pool[0])} of {len(server.tables.ring)}")
    for i, tokens in enumerate(answers[:4]):
        print(f"request {i}: {tokens[:12]}")


if __name__ == "__main__":
    main()
