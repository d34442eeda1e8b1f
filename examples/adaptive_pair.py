"""Two small decoders with random weights generate together under the entropy gate.

What a serving loop around this library looks like: each model keeps a paged key/value cache of its
own; after every gate step a sequence's next token is produced by whichever model the gate chose.
A model that was just switched to has not seen the tokens the other one produced, so it brings
them all in one chunk, while the sequences that stayed bring one token each; both kinds are one call of
``ead_kv_write`` and ``ead_kv_attention``.  The final norm's output goes straight into ``ead_step``.

With ``--rope`` query and key heads are normalised and rotated on their way into the cache (``ead_kv_rotate_write``); with ``--w8``
all products run in 8 bits (``ead_linear`` on weights with a scale per 128 x 128, on activations as the norm and ``ead_quantise``
write them).  At the end each model says what it thinks of the tokens that were produced (``ead_token_logprobs``).

    python examples/adaptive_pair.py [--steps 40] [--e4m3] [--rope] [--w8]
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

    def __init__(self, seed, V, hidden, heads_q, heads_kv, dim, layers, B, max_len, e4m3=False, window=0, sinks=0, rope=False, w8=False):
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
        self.rope = self.w8 = None
        if rope:
            inv_freq = (10000.0 ** -(torch.arange(0, dim, 2, dtype=torch.float64) / dim)).float().cuda()
            self.rope = [E.ead_rope(inv_freq, dim, q_weight=1 + 0.1 * w(dim), k_weight=1 + 0.1 * w(dim)) for _ in range(layers)]
        if w8:
            self.w8 = [{k: to_8_bits(l[k]) for k in ("qkv", "out", "up", "down")} for l in self.layers]
            self.head8 = to_8_bits(self.head)
        self.cached = [0] * B                      # tokens of each sequence that are in the cache
        self.workspace = torch.zeros(E.EAD_KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
        self.score_space = torch.zeros(E.EAD_LOGPROB_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def forget(self):
        self.cached = [0] * self.B

    def step(self, history, rows):
        """Brings the sequences in `rows` up to date with `history` (a list of token lists); final hidden states
        of their last tokens in a [B, hidden] tensor (zeros elsewhere)."""
        x, starts, new = self.run(history, rows)
        hidden = torch.zeros(self.B, self.hidden, dtype=torch.bfloat16, device="cuda")
        last = [b for b in range(self.B) if new[b]]
        hidden[last] = x[(starts[1:][last] - 1).cuda()]
        return hidden

    def score(self, history):
        """What this model thinks of every token of `history` but the first ones, in one pass over whole sequences: log probabilities, ranks and
        entropies, sequence by sequence."""
        self.forget()
        x, starts, _ = self.run(history, set(range(self.B)))
        logits = torch.empty(len(x), self.head.shape[0], device="cuda")
        if self.w8:
            E.ead_linear(quantised(x, 128), self.head8, logits, stream=E.current_stream())
        else:
            logits.copy_(x @ self.head.T)
        nxt = [t for h in history for t in h[1:] + [-1]]                  # the last position has no token to score
        n = len(nxt)
        out = dict(logprob=torch.empty(n, device="cuda"), entropy=torch.empty(n, device="cuda"), rank=torch.empty(n, dtype=torch.int32, device="cuda"))
        E.ead_token_logprobs(logits, torch.tensor(nxt, dtype=torch.int32, device="cuda"), **out, workspace=self.score_space, status=self.status,
                             stream=E.current_stream())
        return {k: [v[starts[b]:starts[b + 1] - 1].tolist() for b in range(self.B)] for k, v in out.items()}

    def run(self, history, rows):
        """The sequences' new tokens through the layers: normalised final states of all of them, where each sequence's begin, and the tokens."""
        new = [history[b][self.cached[b]:] if b in rows else [] for b in range(self.B)]
        tokens = torch.tensor([t for n in new for t in n], dtype=torch.long, device="cuda")
        starts = torch.tensor([0] + [len(n) for n in new]).cumsum(0).int()
        lens = [self.cached[b] + len(new[b]) for b in range(self.B)]
        batch = E.ead_kv_batch(self.table, starts.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), n_tokens=len(tokens),
                               max_new=max(len(n) for n in new), max_len=max(lens))
        stream = torch.cuda.current_stream().cuda_stream
        D, hq, hk = self.dim, self.heads_q, self.heads_kv
        n = len(tokens)
        stream_x = self.embed[tokens]              # the residual stream
        x = torch.empty_like(stream_x)
        x8 = quantised(x, E.EAD_FMT_BLOCK, fill=False) if self.w8 else None
        add, residual = stream_x, None             # what the next norm adds to the stream

        def norm(weight):
            """The next norm, and what the following product takes of it."""
            if not self.w8:
                E.ead_add_rmsnorm(add, weight, x, residual=residual, residual_out=stream_x, stream=stream)
                return x
            E.ead_add_rmsnorm(add, weight, x8.held[0], residual=residual, residual_out=stream_x, out_scale=x8.held[1], stream=stream)
            return x8

        def product(x, layer, name):
            if not self.w8:
                return x @ self.layers[layer][name].T
            out = torch.empty(n, self.w8[layer][name].rows, dtype=torch.bfloat16, device="cuda")
            E.ead_linear(x, self.w8[layer][name], out, status=self.status, stream=stream)
            return out

        for l, (layer, cache) in enumerate(zip(self.layers, self.caches)):
            qkv = product(norm(layer["norm1"]), l, "qkv").view(n, hq + 2 * hk, D)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]           # slices of one projection, as they are
            if self.rope:
                E.ead_kv_rotate_write(self.rope[l], cache, batch, q, k, v, q, status=self.status, stream=stream)
            else:
                E.ead_kv_write(cache, batch, k, v, status=self.status, stream=stream)
            out = torch.empty(n, hq, D, dtype=torch.bfloat16, device="cuda")
            E.ead_kv_attention(cache, batch, q, out, scale=D ** -0.5, window=self.window, sinks=self.sinks,
                               workspace=self.workspace, status=self.status, stream=stream)
            out = out.view(n, -1)
            add, residual = product(quantised(out, 128) if self.w8 else out, l, "out"), stream_x
            gate, up = product(norm(layer["norm2"]), l, "up").chunk(2, -1)
            add = product(quantised(up, 128, gate) if self.w8 else torch.nn.functional.silu(gate) * up, l, "down")
        E.ead_add_rmsnorm(add, self.final, x, residual=residual, stream=stream)
        self.cached = lens
        return x, starts, new


def quantised(x, block, gate=None, fill=True):
    """8-bit rows of x (times silu(gate)) with a scale per `block` values; with `fill` false the place for them."""
    n, cols = x.shape
    m = E.ead_e4m3_matrix(torch.empty(n, cols, dtype=torch.uint8, device="cuda"),
                          torch.empty(n, -(-cols // block), dtype=torch.uint8, device="cuda"), block=(1, block))
    if fill:
        E.ead_quantise(x, m, gate=gate, stream=E.current_stream())
    return m


def to_8_bits(w):
    """Weights with a scale per 128 x 128."""
    rows, cols = w.shape
    m = E.ead_e4m3_matrix(torch.empty(rows, cols, dtype=torch.uint8, device="cuda"),
                          torch.empty(-(-rows // 128), -(-cols // 128), dtype=torch.uint8, device="cuda"), block=(128, 128))
    E.ead_quantise(w, m, stream=E.current_stream())
    return m


def generate(steps=40, B=6, V=512, prompt=12, tau=5.75, e4m3=False, seed=0, small_kw={}, large_kw={}, rope=False, w8=False):
    """Returns the token histories, which model produced each token ([steps, B]) and the two decoders."""
    max_len = prompt + steps
    small = Decoder(seed + 1, V, 256, 4, 2, 64, 2, B, max_len, e4m3, rope=rope, w8=w8, **small_kw)
    large = Decoder(seed + 2, V, 512, 8, 2, 64, 3, B, max_len, e4m3, rope=rope, w8=w8, **large_kw)
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
    ap.add_argument("--rope", action="store_true", help="norm and rotation of query and key heads")
    ap.add_argument("--w8", action="store_true", help="products in 8 bits")
    a = ap.parse_args()
    history, log, small, large = generate(steps=a.steps, e4m3=a.e4m3, rope=a.rope, w8=a.w8)
    for b, h in enumerate(history):
        print(f"sequence {b}: models {''.join('SL'[row[b]] for row in log)}  last tokens {h[-6:]}")
    switches = sum(log[t][b] != log[t - 1][b] for t in range(1, len(log)) for b in range(len(history)))
    print(f"{switches} switches, large-model share {sum(map(sum, log)) / (len(log) * len(history)):.2f}, "
          f"status {small.status.item() | large.status.item():#x}")
    for name, m in (("small", small), ("large", large)):
        own, other = [], []
        for b, scores in enumerate(m.score(history)["logprob"]):
            for t, lp in enumerate(scores[-a.steps:]):
                (own if log[t][b] == (m is large) else other).append(lp)
        mean = lambda v: f"{sum(v) / len(v):.2f}" if v else "-"           # noqa: E731
        print(f"{name} model: mean log probability of its own tokens {mean(own)}, of the other's {mean(other)}")


if __name__ == "__main__":
    main()
