"""A decode loop over a paged cache that evicts: the calls of the library as a
serving program makes them.

A synthetic decoder (random weights, random token embeddings, attention and
residual only) runs a prompt and then generates, for a batch of sequences:

  per layer   epikv_append    rotate the token's queries and keys, write keys
                              and values into the cache's pages (bf16 or 4 bits)
              epikv_attend    attention of the queries over the pages
  per token   epikv_score_tokens   the token's frozen score from the band layers
  every N     epikv_evict_step     keep the prompt, the latest and the best
                                   scored tokens, in the sequence's own pages

Nothing in the loop waits for the device: lengths and positions stay there.

    python examples/decode_evict.py [--format bf16|mxfp4] [--tokens 256] ...
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_26472_amd import epikv as E  # noqa: E402


def check_positions(prompt, tokens, max_positions):
    """A token past the table would be left out of the cache."""
    if prompt + tokens > max_positions:
        raise ValueError(f"{prompt} + {tokens} tokens, the positions' table holds {max_positions}")


class Decoder:
    """The loop's state: weights, cache, page table, lengths, scores."""

    def __init__(self, batch=4, layers=4, hidden=1024, heads=8, kv_heads=2, head_dim=128, page=16, prompt=100,
                 budget=256, every=64, fmt="bf16", theta=500000.0, max_positions=4096, seed=0, history=False):
        if layers < 2:
            raise ValueError("the scores need two layers at least, one of each band")
        if not 1 <= prompt <= max_positions:
            raise ValueError(f"a prompt of 1 to {max_positions} tokens (the positions' table)")
        dev = self.dev = torch.device("cuda")
        g = self.gen = torch.Generator(device=dev).manual_seed(seed)
        self.B, self.L, self.D, self.Hq, self.H, self.d = batch, layers, hidden, heads, kv_heads, head_dim
        self.prompt, self.every, self.max_positions = prompt, every, max_positions
        self.cfg = E.default_cfg(batch=batch, hidden=hidden, n_layers=layers, n_kv_heads=kv_heads,
                                 head_dim=head_dim, page_size=page, n_band_a=1, n_band_b=1, budget=budget,
                                 kv_format=E.KV_MXFP4 if fmt == "mxfp4" else E.KV_BF16)
        self.bands = (layers // 3, 2 * layers // 3)  # the layers scored: A, B
        self.rope = E.default_rope(rotary_dim=head_dim, n_pos=max_positions, theta=theta)
        self.table = torch.empty(E.rope_table_bytes(self.rope) // 4, device=dev)
        E.epikv_rope_table(self.rope, self.table)

        def weight(n, m):
            return (torch.randn(n, m, generator=g, device=dev) / n ** 0.5).bfloat16()
        self.wqkv = [weight(hidden, (heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.wo = [weight(heads * head_dim, hidden) for _ in range(layers)]

        # a sequence never holds more than its budget and one interval (or its prompt)
        self.room = max(budget, prompt) + every
        self.width = -(-self.room // page)
        row = E.kv_row_bytes(self.cfg)
        self.pages = torch.zeros(layers, 2, batch * self.width, page, row, dtype=torch.uint8, device=dev)
        self.pool = E.pool_of(self.pages)
        self.page_table = torch.randperm(batch * self.width, generator=g, device=dev).int().view(batch, -1)

        def ints(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=dev)
        self.n_cached, self.position = ints(batch), ints(batch)
        self.n_prefix = torch.full((batch,), prompt, dtype=torch.int32, device=dev)
        self.pos, self.scores = ints(batch, self.room), torch.zeros(batch, self.room, device=dev)
        self.keep, self.n_keep, self.status = ints(batch, budget), ints(batch), ints(batch)
        self.state = torch.zeros(2, E.state_bytes(self.cfg), dtype=torch.uint8, device=dev)
        for s in self.state:
            E.epikv_state_init(self.cfg, s)
        nbytes = max(E.workspace_bytes(self.cfg, 0), E.attend_workspace_bytes(self.cfg, 1, heads),
                     E.attend_workspace_bytes(self.cfg, prompt, heads))
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        self.evict_io = E.make_step_io(
            0, None, 0, 0, self.n_cached, self.n_prefix, self.pool, self.page_table, self.width, E.Pool(), None, 0,
            self.scores, self.room, None, None, self.keep, self.n_keep, self.status, self.workspace,
            nbytes, src_pos=self.pos, dst_pos=self.pos, in_place=E.COMPACT_IN_PLACE)
        self.tokens = 0
        # for a check only: everything ever appended, by position
        self.history = [[] for _ in range(layers)] if history else None
        self.last = None

    def feed(self, x):
        """x [batch][chunk][hidden]: through every layer; returns the output."""
        B, C, _ = x.shape
        self.n_cached += C
        hidden = []
        self.last = []
        for l in range(self.L):
            qkv = (x @ self.wqkv[l]).view(B, C, self.Hq + 2 * self.H, self.d)
            q, k, v = qkv.split([self.Hq, self.H, self.H], 2)
            out = torch.empty(B, C, self.Hq, self.d, dtype=x.dtype, device=self.dev)
            if self.history is not None:
                self.history[l].append((k.float().clone(), v.float().clone(), self.position.clone()))
            E.epikv_append(self.cfg, E.make_append_io(
                C, self.pool, l, self.page_table, self.width, self.n_cached, k, v, rope=self.rope,
                table=self.table, positions=self.position, q=q, q_out=q, pos=self.pos, ld_s=self.room,
                seq_status=self.status))
            E.epikv_attend(self.cfg, E.make_attend_io(
                C, self.pool, l, self.page_table, self.width, self.n_cached, q, out, seq_status=self.status,
                workspace=self.workspace, workspace_bytes_=self.workspace.numel()))
            if self.history is not None:
                self.last.append((q.clone(), out.clone()))
            x = x + out.view(B, C, -1) @ self.wo[l]
            if l in self.bands:
                hidden.append(x)
        self.position += C
        self._score(hidden, C)
        return x

    def _score(self, hidden, chunk):
        """Scores of the chunk's tokens, 64 at most a call."""
        done = self.n_cached - chunk
        for a in range(0, chunk, 64):
            n = min(64, chunk - a)
            E.epikv_score_tokens(self.cfg, n, [h[:, a:] for h in hidden], self.D, hidden[0].stride(0),
                                 done + (a + n), self.state[0], self.state[1], self.scores, self.room)
            self.state = self.state.flip(0)

    def evict(self):
        E.epikv_evict_step(self.cfg, self.evict_io)
        self.n_cached.copy_(self.n_keep)

    def run(self, n_tokens):
        check_positions(self.prompt, self.tokens + n_tokens, self.max_positions)
        def embed(n):
            return torch.randn(self.B, n, self.D, generator=self.gen, device=self.dev).bfloat16()
        if self.tokens == 0:
            self.feed(embed(self.prompt))
        for _ in range(n_tokens):
            if self.tokens and self.tokens % self.every == 0:
                self.evict()
            x = self.feed(embed(1))
            self.tokens += 1
        return x


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--format", choices=["bf16", "mxfp4"], default="bf16")
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--prompt", type=int, default=100)
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--budget", type=int, default=256)
    p.add_argument("--every", type=int, default=64)
    p.add_argument("--max-positions", type=int, default=4096)
    a = p.parse_args(argv)
    warm = min(a.tokens, a.every)
    check_positions(a.prompt, warm + a.tokens, a.max_positions)
    m = Decoder(batch=a.batch, layers=a.layers, prompt=a.prompt, budget=a.budget, every=a.every, fmt=a.format,
                max_positions=a.max_positions)
    m.run(warm)
    torch.cuda.synchronize()
    start = time.perf_counter()
    m.run(a.tokens)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - start
    held = m.n_cached.tolist()
    assert not m.status.any().item(), m.status.tolist()
    print(f"{a.tokens} tokens of {a.batch} sequences in {seconds:.3f} s "
          f"({1e6 * seconds / a.tokens:.0f} us a token); {m.position[0].item()} positions seen, "
          f"{held} held in {a.format} rows of {E.kv_row_bytes(m.cfg)} bytes")


if __name__ == "__main__":
    main()
