"""Two small decoders with random weights generate together under the entropy gate.

What a serving loop around this library looks like: each model keeps a paged key/value cache of its
own; after every gate step a sequence's next token is produced by whichever model the gate chose.
A model that was just switched to has not seen the tokens the other one produced, so it brings
them all in one chunk, while the sequences that stayed bring one token each; both kinds are one call of
``ead_kv_write`` and ``ead_kv_attention``.  The final norm's output goes straight into ``ead_step``.

    python examples/adaptive_pair.py [--steps 40] [--e4m3]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2502_06833_b200 import binding as E

PAGE = 16


class Decoder:
    """A pre-norm decoder (attention and a gated MLP per layer) over this library's cache operators."""

    def __init__(self, seed, V, hidden, heads_q, heads_kv, dim, layers, B, max_len, e4m3=False, window=0, sinks=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *shape: (torch.randn(*shape, device="cuda", generator=g) * shape[-1] ** -0.5).bfloat16()   # noqa: E731
        self.B, self.hidden, self.heads_q, self.heads_kv, self.dim = B, hidden, heads_q, heads_kv, dim
        self.window, self.sinks = window, sinks
        self.embed = torch.randn(V, hidden, device="cuda", generator=g).bfloat16()
        self.head = w(V, hidden)
        self.layers = [dict(qkv=w((heads_q + 2 * heads_kv) * dim, hidden), out=w(hidden, heads_q * dim), up=w(4 * hidden, hidden),
                            down=w(hidden, 2 * hidden), norm1=1 + 0.1 * w(hidden), norm2=1 + 0.1 * w(hidden)) for _ in range(layers)]
        self.final = 1 + 0.1 * w(hidden)
        # one page pool per layer; the pages of a sequence are the same in all of them, handed out in shuffled order
        per = -(-max_len // PAGE)
        self.table = torch.randperm(B * per, generator=torch.Generator().manual_seed(seed)).int().view(B, per).cuda()
        shape = (B * per, heads_kv, PAGE, dim)
        self.caches = []
        for _ in range(layers):
            if e4m3:
                pool = [torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in "kv"]
                scale = [torch.zeros(*shape[:3], dim // E.EAD_FMT_BLOCK, dtype=torch.uint8, device="cuda") for _ in "kv"]
                self.caches.append(E.ead_kv_cache(*pool, *scale))
            else:
                self.caches.append(E.ead_kv_cache(*[torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in "kv"]))
        self.cached = [0] * B                      # tokens of each sequence that are in the cache
        self.workspace = torch.zeros(E.EAD_KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def forget(self):
        self.cached = [0] * self.B

    def step(self, history, rows):
        """Brings the sequences in `rows` up to date with `history` (a list of token lists); final hidden states
        of their last tokens in a [B, hidden] tensor (zeros elsewhere)."""
        new = [history[b][self.cached[b]:] if b in rows else [] for b in range(self.B)]
        tokens = torch.tensor([t for n in new for t in n], dtype=torch.long, device="cuda")
        starts = torch.tensor([0] + [len(n) for n in new]).cumsum(0).int()
        lens = [self.cached[b] + len(new[b]) for b in range(self.B)]
        batch = E.ead_kv_batch(self.table, starts.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), n_tokens=len(tokens),
                               max_new=max(len(n) for n in new), max_len=max(lens))
        stream = torch.cuda.current_stream().cuda_stream
        D, hq, hk = self.dim, self.heads_q, self.heads_kv
        stream_x = self.embed[tokens]              # the residual stream
        x = torch.empty_like(stream_x)
        add, residual = stream_x, None             # what the next norm adds to the stream
        for layer, cache in zip(self.layers, self.caches):
            E.ead_add_rmsnorm(add, layer["norm1"], x, residual=residual, residual_out=stream_x, stream=stream)
            qkv = (x @ layer["qkv"].T).view(len(tokens), hq + 2 * hk, D)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]           # slices of one projection, as they are
            E.ead_kv_write(cache, batch, k, v, status=self.status, stream=stream)
            out = torch.empty(len(tokens), hq, D, dtype=torch.bfloat16, device="cuda")
            E.ead_kv_attention(cache, batch, q, out, scale=D ** -0.5, window=self.window, sinks=self.sinks,
                               workspace=self.workspace, status=self.status, stream=stream)
            E.ead_add_rmsnorm(out.view(len(tokens), -1) @ layer["out"].T, layer["norm2"], x, residual=stream_x, residual_out=stream_x,
                              stream=stream)
            gate, up = (x @ layer["up"].T).chunk(2, -1)
            add, residual = (torch.nn.functional.silu(gate) * up) @ layer["down"].T, stream_x
        E.ead_add_rmsnorm(add, self.final, x, residual=residual, stream=stream)
        self.cached = lens
        hidden = torch.zeros(self.B, self.hidden, dtype=torch.bfloat16, device="cuda")
        last = [b for b in range(self.B) if new[b]]
        hidden[last] = x[(starts[1:][last] - 1).cuda()]
        return hidden


def generate(steps=40, B=6, V=512, prompt=12, tau=5.75, e4m3=False, seed=0, small_kw={}, large_kw={}):
    """Returns the token histories, which model produced each token ([steps, B]) and the two decoders."""
    max_len = prompt + steps
    small = Decoder(seed + 1, V, 256, 4, 2, 64, 2, B, max_len, e4m3, **small_kw)
    large = Decoder(seed + 2, V, 512, 8, 2, 64, 3, B, max_len, e4m3, **large_kw)
    g = torch.Generator().manual_seed(seed)
    history = [torch.randint(0, V, (prompt,), generator=g).tolist() for _ in range(B)]
    ctx = E.ead_create(B=B, V=V, H_small=256, H_large=512, w=3, d_min=4, tau=tau, W_small=small.head, W_large=large.head,
                       device=torch.cuda.current_device(), stream=torch.cuda.current_stream().cuda_stream)
    tok = torch.empty(B, dtype=torch.int32, device="cuda")
    used, nxt = (torch.empty(B, dtype=torch.uint8, device="cuda") for _ in range(2))
    active, log = [0] * B, []
    for _ in range(steps):
        h = [m.step(history, {b for b in range(B) if active[b] == k}) if k in active else
             torch.zeros(B, m.hidden, dtype=torch.bfloat16, device="cuda") for k, m in enumerate((small, large))]
        E.ead_step(ctx, h[0], h[1], tok, None, None, used, nxt)
        for b, t in enumerate(tok.tolist()):
            history[b].append(t)
        log.append(used.tolist())
        active = nxt.tolist()
    E.ead_status(ctx)
    E.ead_destroy(ctx)
    return history, log, small, large


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--e4m3", action="store_true", help="8-bit caches")
    a = ap.parse_args()
    history, log, small, large = generate(steps=a.steps, e4m3=a.e4m3)
    for b, h in enumerate(history):
        print(f"sequence {b}: models {''.join('SL'[row[b]] for row in log)}  last tokens {h[-6:]}")
    switches = sum(log[t][b] != log[t - 1][b] for t in range(1, len(log)) for b in range(len(history)))
    print(f"{switches} switches, large-model share {sum(map(sum, log)) / (len(log) * len(history)):.2f}, "
          f"status {small.status.item() | large.status.item():#x}")


if __name__ == "__main__":
    main()
