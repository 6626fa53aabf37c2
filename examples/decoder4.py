"""A small decoder whose weights and cache are held in 4 bits, on the library's
decoder operators: every projection is w4_matvec; a prompt goes through
kv4_append and prompt_attention, which sees keys and values as the cache holds
them; each further token through kv4_append and kv4_attention, the whole step
one HIP graph.  Random weights.

    python examples/decoder4.py --batch 8 --prompt 300 --tokens 64
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np  # noqa: E402
import torch  # noqa: E402

import paper_2209_12982_amd as W  # noqa: E402


class Decoder:
    """`sequences` sequences of up to `capacity` tokens each."""

    def __init__(self, sequences, capacity, layers=2, hidden=512, heads=8, kv_heads=2, head_dim=64, inner=1024, vocab=2048,
                 page=64, dtype=torch.bfloat16, seed=0):
        rng = np.random.default_rng(seed)
        self.heads, self.kv_heads, self.dim, self.dtype, self.page = heads, kv_heads, head_dim, dtype, page

        def weights(n, k):
            w = rng.normal(0, k ** -0.5, (n, k)).astype(np.float32)
            return tuple(torch.from_numpy(a).cuda() for a in W.w4_quantize_weights(w))

        self.embedding = torch.from_numpy(rng.normal(0, 1, (vocab, hidden)).astype(np.float32)).to(dtype).cuda()
        self.layers = [dict(qkv=weights((heads + 2 * kv_heads) * head_dim, hidden), out=weights(hidden, heads * head_dim),
                            up=weights(2 * inner, hidden), down=weights(hidden, inner)) for _ in range(layers)]
        self.head = weights(vocab, hidden)

        # the cache: each sequence's pages, given out in random order
        per = -(-capacity // page)
        order = rng.permutation(sequences * per).astype(np.int32).reshape(sequences, per)
        self.table = torch.from_numpy(order).cuda()
        widths = (head_dim // 2, head_dim // 32) * 2
        self.caches = [tuple(torch.zeros((sequences * per, kv_heads, page, w), dtype=torch.uint8, device="cuda")
                             for w in widths) for _ in range(layers)]
        self.lens = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.capacity, self.longest = per * page, 0         # tokens of a sequence: the table's, and held by the longest
        angle = np.arange(per * page)[:, None] * 10000.0 ** (-np.arange(0, head_dim, 2) / head_dim)
        self.cos_sin = torch.from_numpy(np.concatenate((np.cos(angle), np.sin(angle)), -1).astype(np.float32)).cuda()

        shapes = [(v[0].shape[0], v[0].shape[1] * 2) for layer in self.layers for v in layer.values()]
        need = max(W.w4_matvec_workspace_bytes(sequences, n, k) for n, k in shapes + [(vocab, hidden)])
        need = max(need, W.kv4_attention_workspace_bytes(sequences, 1, heads, kv_heads, head_dim, per, page))
        self.workspace = torch.empty(need + 16, dtype=torch.uint8, device="cuda")

    def _product(self, x, weights):
        y = torch.empty((x.shape[0], weights[0].shape[0]), dtype=x.dtype, device="cuda")
        # a prompt's many rows get along without room for parts
        W.w4_matvec(x, *weights, y, workspace=self.workspace if x.shape[0] == self.table.shape[0] else None)
        return y

    @staticmethod
    def _norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def _forward(self, tokens, positions, slots, attend):
        """Logits of `tokens`; attend(layer, q, k, v, out) is the attention of rotated queries."""
        x = self.embedding[tokens]
        rows, hq, hkv, d = len(tokens), self.heads, self.kv_heads, self.dim
        q_out = torch.empty((rows, hq, d), dtype=self.dtype, device="cuda")
        k_out, v_out = (torch.empty((rows, hkv, d), dtype=self.dtype, device="cuda") for _ in range(2))
        out = torch.empty_like(q_out)
        for layer, weights in enumerate(self.layers):
            qkv = self._product(self._norm(x), weights["qkv"]).view(rows, hq + 2 * hkv, d)
            q, k, v = qkv.split((hq, hkv, hkv), 1)
            W.kv4_append(q, k, v, self.cos_sin, positions, slots, self.caches[layer], q_out, k_out, v_out,
                         values=W.KV4_CACHED)
            attend(layer, q_out, k_out, v_out, out)
            x = x + self._product(out.view(rows, hq * d), weights["out"])
            gate, up = self._product(self._norm(x), weights["up"]).chunk(2, -1)
            x = x + self._product(torch.nn.functional.silu(gate) * up, weights["down"])
        return self._product(self._norm(x), self.head)

    def _room(self, longest):
        """Refuses what the table has no pages for: an index past it would be one past its memory."""
        if longest > self.capacity:
            raise ValueError(f"{longest} tokens in a sequence, the cache holds {self.capacity}")
        self.longest = longest

    def prompt(self, prompts):
        """Fills the cache with the prompts (lists of tokens, one a sequence) and
        returns the logits of all their tokens [total, vocab]."""
        counts = [len(p) for p in prompts]
        if len(counts) != len(self.lens):
            raise ValueError(f"{len(counts)} prompts for {len(self.lens)} sequences")
        self._room(max(counts))
        tokens = torch.tensor([t for p in prompts for t in p], dtype=torch.int64, device="cuda")
        at = torch.tensor([i for n in counts for i in range(n)], dtype=torch.int64, device="cuda")
        seq = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts)).cuda()
        slots = self.table[seq, at // self.page].long() * self.page + at % self.page
        cu = torch.tensor(np.cumsum([0] + counts), dtype=torch.int32, device="cuda")

        def attend(layer, q, k, v, out):
            W.prompt_attention(q, k, v, cu, cu, max(counts), out, self.dim ** -0.5)
        self.lens.copy_(torch.tensor(counts, dtype=torch.int32))
        return self._forward(tokens, at.to(torch.int32), slots, attend)

    def step(self, tokens):
        """Appends one token to each sequence; returns their logits [sequences, vocab]."""
        self._room(self.longest + 1)
        at = self.lens.long()
        slots = self.table.gather(1, (at // self.page)[:, None])[:, 0].long() * self.page + at % self.page
        positions = self.lens.clone()
        self.lens += 1

        def attend(layer, q, k, v, out):
            W.kv4_attention(q, self.caches[layer], self.table, self.lens, out, self.dim ** -0.5, workspace=self.workspace)
        return self._forward(tokens, positions, slots, attend)

    def capture(self):
        """step() as a HIP graph: returns a function with the same arguments."""
        tokens, held, longest = torch.zeros_like(self.lens, dtype=torch.int64), self.lens.clone(), self.longest
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                       # once outside of the graph: what is laid out at the first use
            self.step(tokens)
        torch.cuda.current_stream().wait_stream(side)
        self.lens.copy_(held)                               # the token written there is overwritten by the next one
        self.longest = longest
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            logits = self.step(tokens)
        self.longest = longest                              # nothing has run: a replay counts its token

        def replay(new):
            self._room(self.longest + 1)
            tokens.copy_(new)
            graph.replay()
            return logits
        return replay


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("batch", 8), ("prompt", 300), ("tokens", 64), ("layers", 4), ("hidden", 2048), ("heads", 16),
                        ("kv-heads", 4), ("head-dim", 128), ("inner", 4096), ("vocab", 8192)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args()
    model = Decoder(a.batch, a.prompt + a.tokens + 1, a.layers, a.hidden, a.heads, a.kv_heads, a.head_dim, a.inner, a.vocab)
    rng = np.random.default_rng(1)
    lens = [int(n) for n in rng.integers(max(1, a.prompt // 2), a.prompt + 1, a.batch)]
    prompts = [rng.integers(0, a.vocab, n).tolist() for n in lens]
    for _ in range(2):                                      # the second time is measured
        torch.cuda.synchronize()
        start = time.perf_counter()
        logits = model.prompt(prompts)
        torch.cuda.synchronize()
        took = time.perf_counter() - start
    print(f"prompt: {sum(lens)} tokens of {a.batch} sequences in {took * 1e3:.2f} ms")
    new = logits[torch.tensor(np.cumsum(lens) - 1, device="cuda")].argmax(-1)
    step = model.capture()
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(a.tokens):
        new = step(new).argmax(-1)
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    print(f"decoding: {a.tokens} steps of {a.batch} tokens, {took / a.tokens * 1e6:.0f} us a step, "
          f"{a.batch * a.tokens / took:.0f} tokens/s")


if __name__ == "__main__":
    main()
