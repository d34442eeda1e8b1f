"""Cases of the decoder-side operators that stand around the gate step, with their plain forms.

The gate step starts from the final hidden states of two decoders.  The operators here are what
such a decoder does with its context: it adds the last block's output to the residual stream and
normalises it (``norm``), writes the new tokens' keys and values into a paged cache, quantised or
not (``write``), attends from the new tokens over that cache (``attention``), and hands a
sequence's context out again (``read``).  A sequence that stays on its model brings one new token
per step; one that was just switched brings all the tokens it missed.

With ``own`` false, ``run`` is the plain form: elementary torch operations in 32 bits, rounded once
at the end.  With ``own`` true it calls the library's entry points.

8-bit values are e4m3 with one power-of-two scale per 32 consecutive values: the smallest power
for which no finite value of the block exceeds 448, kept between 2^-120 and 2^119 and stored as
its exponent plus 127.
"""
import random

import torch

own = False

_GROUP = 32                      # values that share one scale
_WORKSPACE = 64 << 20            # bytes; what the attention entry point asks for


# ----------------------------------------------------------------------------- cases
def listed():
    return [
        # one sequence at single-token decoding on a small model (2048 = 32 x 64): pure latency
        dict(name="attention_one_sequence", op="attention", fmt="bf16", B=1, new_lo=1, new_hi=1, chunk_share=0.0,
             len_lo=777, len_hi=777, heads_q=32, heads_kv=8, dim=64, page=16, window=0, sinks=0),
        # a full batch of single-token decoding on the LLaMA-shaped large model (4096 = 32 x 128)
        dict(name="attention_single_tokens", op="attention", fmt="bf16", B=64, new_lo=1, new_hi=1, chunk_share=0.0,
             len_lo=1024, len_hi=8192, heads_q=32, heads_kv=8, dim=128, page=64, window=0, sinks=0),
        # long contexts kept in 8 bits on the Qwen-shaped large model (5120 = 40 x 128), one token each
        dict(name="attention_long_e4m3", op="attention", fmt="e4m3", B=24, new_lo=1, new_hi=1, chunk_share=0.0,
             len_lo=4001, len_hi=32001, heads_q=40, heads_kv=8, dim=128, page=32, window=0, sinks=0),
        # a step in which a quarter of the rows was just switched and catches up on 10 to 200 tokens
        dict(name="attention_hand_over", op="attention", fmt="bf16", B=32, new_lo=10, new_hi=200, chunk_share=0.25,
             len_lo=501, len_hi=6001, heads_q=40, heads_kv=8, dim=128, page=16, window=0, sinks=0),
        # chunks of long prompts over their earlier chunks: the compute-bound end
        dict(name="attention_prompt_chunks", op="attention", fmt="bf16", B=2, new_lo=2041, new_hi=2048, chunk_share=1.0,
             len_lo=6007, len_hi=8192, heads_q=32, heads_kv=8, dim=128, page=64, window=0, sinks=0),
        # long prompts of a small Qwen-shaped model (1536 = 12 x 128) with a window and four sinks, 8-bit cache
        dict(name="attention_window_e4m3", op="attention", fmt="e4m3", B=4, new_lo=700, new_hi=1300, chunk_share=1.0,
             len_lo=4003, len_hi=12003, heads_q=12, heads_kv=2, dim=128, page=16, window=1024, sinks=4),
        # one step's keys and values of a batch, unquantised
        dict(name="write_step", op="write", fmt="bf16", B=64, new_lo=1, new_hi=1, chunk_share=0.0,
             len_lo=100, len_hi=2000, heads_q=32, heads_kv=8, dim=128, page=16, window=0, sinks=0),
        # prompts written into an 8-bit cache
        dict(name="write_prompts_e4m3", op="write", fmt="e4m3", B=12, new_lo=1500, new_hi=2600, chunk_share=1.0,
             len_lo=2600, len_hi=4100, heads_q=40, heads_kv=8, dim=128, page=32, window=0, sinks=0),
        # a short prefix read back for another sequence
        dict(name="read_prefix", op="read", fmt="e4m3", B=1, new_lo=509, new_hi=509, chunk_share=1.0,
             len_lo=600, len_hi=600, heads_q=12, heads_kv=2, dim=128, page=16, window=0, sinks=0),
        # whole contexts read back, as when sequences leave the GPU
        dict(name="read_contexts_e4m3", op="read", fmt="e4m3", B=16, new_lo=5001, new_hi=8001, chunk_share=1.0,
             len_lo=8001, len_hi=8190, heads_q=40, heads_kv=8, dim=128, page=32, window=0, sinks=0),
        # the final norm of one decoding step (its output feeds the gate step)
        dict(name="norm_step", op="norm", fmt="bf16", rows=64, H=4096),
        # a norm inside a prompt's pass whose output goes on in 8 bits
        dict(name="norm_prompt_e4m3", op="norm", fmt="e4m3", rows=16384, H=5120),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    top = {}                                                             # the most work of a listed case, by operator
    for c in listed():
        w = work(c)
        t = top.setdefault(c["op"], {"bytes": 0, "flops": 0})
        t["bytes"], t["flops"] = max(t["bytes"], w["bytes"]), max(t["flops"], w["flops"])
    while True:
        op = rng.choice(["attention", "attention", "attention", "attention", "write", "read", "norm"])
        fmt = rng.choice(["bf16", "e4m3"])
        if op == "norm":
            c = dict(op=op, fmt=fmt, rows=_log_int(rng, 1, 16384), H=rng.choice([1536, 2048, 4096, 5120, 32 * rng.randint(2, 170)]))
        else:
            heads_q, heads_kv, dim = rng.choice([(32, 8, 64), (32, 8, 128), (40, 8, 128), (12, 2, 128), (28, 4, 128), (16, 16, 64)])
            B = _log_int(rng, 1, 64)
            share = rng.choice([0.0, 0.0, 0.25, 1.0]) if op != "read" else 1.0
            new_hi = _log_int(rng, 2, 2600) if share else 1
            new_lo = rng.randint(max(1, new_hi // 3), new_hi) if share else 1
            len_hi = max(new_hi, _log_int(rng, 40, 32001))
            c = dict(op=op, fmt=fmt, B=B, new_lo=new_lo, new_hi=new_hi, chunk_share=share, len_lo=rng.randint(max(new_hi, len_hi // 4), len_hi),
                     len_hi=len_hi, heads_q=heads_q, heads_kv=heads_kv, dim=dim, page=rng.choice([16, 32, 64, 128]), window=0, sinks=0)
            if op == "attention" and rng.random() < 0.3:
                c["window"], c["sinks"] = _log_int(rng, 16, 4096), rng.choice([0, 1, 4, 64])
            if B * len_hi > 800_000:                                     # keeps the cache of a case within a few GB
                continue
            if op == "attention" and B * heads_q * new_hi * len_hi > 1_600_000_000:   # and the plain form's scores
                continue
        w = work(c)
        if w["bytes"] <= top[op]["bytes"] and w["flops"] <= top[op]["flops"]:
            return c


def _lengths(case):
    """New tokens and context length (the new ones included) of every sequence; by the case alone."""
    spread = lambda step, at, b: (b * step + at) % 1.0                   # noqa: E731
    between = lambda lo, hi, u: lo + int(u * (hi - lo + 1))              # noqa: E731
    rows = range(case["B"])
    new = [between(case["new_lo"], case["new_hi"], spread(0.7548776662, 0.11, b)) if spread(0.5698402910, 0.05, b) < case["chunk_share"] else 1
           for b in rows]
    length = [max(new[b], between(case["len_lo"], case["len_hi"], spread(0.6180339887, 0.37, b))) for b in rows]
    return new, length


def _visible(case, n, length):
    """(query, key) pairs of one sequence, and keys seen by any of its queries."""
    window, sinks = case["window"], case["sinks"]
    lo = lambda p: max(0, p - window + 1) if window else 0             # noqa: E731
    first = length - n
    return sum(p + 1 - lo(p) + min(sinks, lo(p)) for p in range(first, length)), length - lo(first) + min(sinks, lo(first))


def work(case):
    if case["op"] == "norm":
        n, H = case["rows"], case["H"]
        out = 2 * H if case["fmt"] == "bf16" else H + H // _GROUP
        return {"bytes": n * (2 * H + 4 * H + out) + 2 * H, "flops": 6 * n * H}
    new, length = _lengths(case)
    heads, dim = case["heads_kv"], case["dim"]
    row = 2 * heads * (2 * dim if case["fmt"] == "bf16" else dim + dim // _GROUP)      # one token's keys and values in the cache
    if case["op"] in ("write", "read"):
        n = sum(new)
        return {"bytes": n * (row + 2 * heads * 2 * dim), "flops": 4 * n * heads * dim}
    pairs, keys = (sum(v) for v in zip(*(_visible(case, n, l) for n, l in zip(new, length))))
    return {"bytes": keys * row + sum(new) * case["heads_q"] * (4 * dim + 4), "flops": 4 * dim * case["heads_q"] * pairs}


# ----------------------------------------------------------------------------- inputs
def _scale_bytes(amax):
    """Stored exponents of the scales for blocks of the given largest magnitudes (32-bit floats)."""
    mant, exp = torch.frexp(amax)                                       # amax = mant * 2^exp, 0.5 <= mant < 1
    k = torch.where(mant > 0.875, exp - 8, exp - 9)                     # 448 = 0.875 * 2^9
    k = torch.where(amax > 0, k.clamp(-120, 119), -120)
    return (k + 127).to(torch.uint8)


def _quantise(x):
    """[..., n] values -> (e4m3 codes, stored scale exponents [..., n / 32])."""
    g = x.unflatten(-1, (-1, _GROUP))
    stored = _scale_bytes(torch.where(torch.isfinite(g), g.abs(), 0.0).amax(-1))
    codes = torch.ldexp(g, 127 - stored.unsqueeze(-1).int()).to(torch.float8_e4m3fn)
    return codes.flatten(-2), stored


def _values(codes, stored):
    g = codes.float().unflatten(-1, (-1, _GROUP))
    return torch.ldexp(g, stored.unsqueeze(-1).int() - 127).flatten(-2)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)   # noqa: E731
    s = dict(case=case)
    if case["op"] == "norm":
        n, H = case["rows"], case["H"]
        channel = torch.exp(0.7 * rnd(H))                                # a few channels carry most of the stream
        s["x"] = (0.5 * rnd(n, H) * channel).bfloat16()
        s["residual_in"] = (2.0 * rnd(n, H) * channel).bfloat16()
        s["residual"] = torch.empty_like(s["residual_in"])
        s["weight"] = (1.0 + 0.2 * rnd(H)).bfloat16()
        s["out"] = torch.empty(n, H, dtype=torch.bfloat16 if case["fmt"] == "bf16" else torch.float8_e4m3fn, device="cuda")
        s["out_scale"] = None if case["fmt"] == "bf16" else torch.empty(n, H // _GROUP, dtype=torch.uint8, device="cuda")
        return s
    B, heads, dim, page = case["B"], case["heads_kv"], case["dim"], case["page"]
    new, length = _lengths(case)
    pages = [-(-l // page) for l in length]
    n_pages, width = sum(pages) + 3, max(pages)
    order = list(range(n_pages))
    random.Random(seed).shuffle(order)                                   # pages in no order, as a pool hands them out
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = torch.tensor(order[at:at + pages[b]], dtype=torch.int32)
        at += pages[b]
    starts = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32)
    s.update(new=new, length=length, total=sum(new), max_new=max(new), max_len=max(length), table=table.cuda(), new_start=starts.cuda(),
             kv_len=torch.tensor(length, dtype=torch.int32).cuda(), status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    channel = torch.exp(0.5 * rnd(heads, 1, dim))                        # keys have strong channels
    for name in ("k", "v"):
        pool = torch.empty(n_pages, heads, page, dim, dtype=torch.bfloat16 if case["fmt"] == "bf16" else torch.float8_e4m3fn, device="cuda")
        scale = None if case["fmt"] == "bf16" else torch.empty(n_pages, heads, page, dim // _GROUP, dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // (heads * page * dim))
        for i in range(0, n_pages, step):
            x = rnd(min(step, n_pages - i), heads, page, dim) * (channel if name == "k" else 1.0)
            x = x.bfloat16()
            if scale is None:
                pool[i:i + step] = x
            else:
                pool[i:i + step], scale[i:i + step] = _quantise(x.float())
        s[name], s[name + "_scale"] = pool, scale
    n = s["total"]
    if case["op"] == "attention":
        s["q"] = (1.5 * rnd(n, case["heads_q"], dim)).bfloat16()
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(n, case["heads_q"], device="cuda")
        s["workspace"] = torch.zeros(_WORKSPACE, dtype=torch.uint8, device="cuda")
    elif case["op"] == "write":
        s["k_new"] = (rnd(n, heads, dim) * channel.squeeze(1)).bfloat16()
        s["v_new"] = rnd(n, heads, dim).bfloat16()
    else:
        s["first"] = torch.tensor([(l - m) // 2 for l, m in zip(length, new)], dtype=torch.int32).cuda()
        s["k_out"] = torch.empty(n, heads, dim, dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    return s


# ----------------------------------------------------------------------------- one pass
def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


def _e8m0(stored):
    return None if stored is None else stored.view(torch.float8_e8m0fnu)


def _own(s):
    from paper_2502_06833_b200 import binding as E
    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "norm":
        E.ead_add_rmsnorm(s["x"], s["weight"], s["out"], residual=s["residual_in"], residual_out=s["residual"], out_scale=s["out_scale"],
                          eps=1e-6, stream=stream)
        return s["out"], _e8m0(s["out_scale"]), s["residual"]
    if "cache" not in s:                                                 # a program describes its cache and its step once
        s["cache"] = E.ead_kv_cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["batch"] = E.ead_kv_batch(s["table"], s["new_start"], s["kv_len"], n_tokens=s["total"], max_new=s["max_new"], max_len=s["max_len"])
    if case["op"] == "attention":
        E.ead_kv_attention(s["cache"], s["batch"], s["q"], s["out"], scale=case["dim"] ** -0.5, window=case["window"], sinks=case["sinks"],
                           lse=s["lse"], workspace=s["workspace"], status=s["status"], stream=stream)
        return s["out"], s["lse"]
    if case["op"] == "write":
        E.ead_kv_write(s["cache"], s["batch"], s["k_new"], s["v_new"], status=s["status"], stream=stream)
        return s["k"], s["v"], _e8m0(s["k_scale"]), _e8m0(s["v_scale"])
    E.ead_kv_read(s["cache"], s["batch"], s["k_out"], s["v_out"], first=s["first"], status=s["status"], stream=stream)
    return s["k_out"], s["v_out"]


def _owners(s):
    """Sequence and index within the sequence's new tokens, for every new token of the step."""
    at = torch.arange(s["total"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["new_start"][1:], at, right=True)
    return b, at - s["new_start"][b]


def _plain_attention(s):
    case = s["case"]
    heads, dim, page, group = case["heads_kv"], case["dim"], case["page"], case["heads_q"] // case["heads_kv"]
    B, N, L = case["B"], s["max_new"], s["max_len"]
    key = torch.arange(L, device="cuda")
    at = s["table"].long()[:, key // page].clamp_min(0)
    k, v = _get(s["k"], s["k_scale"], at, key % page), _get(s["v"], s["v_scale"], at, key % page)      # [B, L, heads, dim]
    b, i = _owners(s)
    q = torch.zeros(B, N, heads, group, dim, device="cuda")
    q[b, i] = s["q"].float().unflatten(1, (heads, group))
    q = q.permute(0, 2, 1, 3, 4).reshape(B, heads, N * group, dim)
    z = (q @ k.permute(0, 2, 3, 1)).mul_(dim ** -0.5).unflatten(2, (N, group))
    new = s["new_start"].diff()
    place = (s["kv_len"] - new)[:, None] + torch.arange(N, device="cuda")               # [B, N]
    seen = key <= place[..., None]
    if case["window"]:
        seen &= (key > place[..., None] - case["window"]) | (key < case["sinks"])
    z.masked_fill_(~seen[:, None, :, None], float("-inf"))
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v.transpose(1, 2)).unflatten(2, (N, group)) / total
    lse = (total.log() + top).squeeze(-1)
    return (o.permute(0, 2, 1, 3, 4)[b, i].flatten(1, 2).to(torch.bfloat16), lse.permute(0, 2, 1, 3)[b, i].flatten(1))


def _put(pool, scale, new, at, slot):
    if scale is None:
        pool[at, :, slot] = new
    else:
        codes, stored = _quantise(new.float())
        pool.view(torch.uint8)[at, :, slot] = codes.view(torch.uint8)
        scale[at, :, slot] = stored


def _get(pool, scale, at, slot):
    """Rows of a pool as 32-bit values."""
    if scale is None:
        return pool[at, :, slot].float()
    return _values(pool.view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn), scale[at, :, slot])


def _plain_write(s):
    page = s["case"]["page"]
    b, i = _owners(s)
    place = (s["kv_len"] - s["new_start"].diff())[b] + i
    at, slot = s["table"][b, place // page].long(), (place % page).long()
    _put(s["k"], s["k_scale"], s["k_new"], at, slot)
    _put(s["v"], s["v_scale"], s["v_new"], at, slot)
    return s["k"], s["v"], _e8m0(s["k_scale"]), _e8m0(s["v_scale"])


def _plain_read(s):
    page = s["case"]["page"]
    b, i = _owners(s)
    place = s["first"][b] + i
    at, slot = s["table"][b, place // page].long(), (place % page).long()
    return _get(s["k"], s["k_scale"], at, slot).to(torch.bfloat16), _get(s["v"], s["v_scale"], at, slot).to(torch.bfloat16)


def _plain_norm(s):
    x = s["x"].float() + s["residual_in"].float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * s["weight"].float()
    if s["case"]["fmt"] == "bf16":
        return y.to(torch.bfloat16), None, x.to(torch.bfloat16)
    codes, stored = _quantise(y)
    return codes, _e8m0(stored), x.to(torch.bfloat16)


_PLAIN = dict(attention=_plain_attention, write=_plain_write, read=_plain_read, norm=_plain_norm)


# ----------------------------------------------------------------------------- in 64 bits
def _exact_codes(x):
    """Block scales and e4m3 values of 64-bit numbers, by logarithms corrected to the definition, and a rounding grid."""
    g = x.unflatten(-1, (-1, _GROUP))
    amax = g.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(amax.clamp_min(2.0 ** -140) / 448.0)).clamp(-120, 119)
    k = torch.where(amax > 448.0 * 2.0 ** k, k + 1, torch.where(amax <= 448.0 * 2.0 ** (k - 1), k - 1, k)).clamp(-120, 119)
    z = g / 2.0 ** k
    step = torch.ldexp(torch.ones_like(z), torch.frexp(z.abs().clamp_min(2.0 ** -6)).exponent - 4)      # spacing of e4m3 at each magnitude
    return (torch.round(z / step) * step).flatten(-2), (2.0 ** k).squeeze(-1)     # round() takes ties to even


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x = s["x"].double() + s["residual_in"].double()
        y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["H"] + 1e-6) * s["weight"].double()
        return (y, None, x) if case["fmt"] == "bf16" else (*_exact_codes(y), x)
    page, dim = case["page"], case["dim"]
    heads, group = case["heads_kv"], case["heads_q"] // case["heads_kv"]
    table = s["table"].cpu()

    def context(name, b, first, last):                                   # [heads, last - first, dim]
        place = torch.arange(first, last)
        at, slot = table[b, place // page].long().cuda(), (place % page).cuda()
        x = s[name].view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).double() if s[name + "_scale"] is not None else s[name][at, :, slot].double()
        if s[name + "_scale"] is not None:
            x = x * (2.0 ** (s[name + "_scale"][at, :, slot].double() - 127)).repeat_interleave(_GROUP, -1)
        return x.transpose(0, 1)

    if case["op"] == "read":
        first = s["first"].tolist()
        parts = [[context(name, b, f, f + n).transpose(0, 1) for b, (f, n) in enumerate(zip(first, s["new"]))] for name in ("k", "v")]
        return tuple(torch.cat(p) for p in parts)
    if case["op"] == "write":
        pools = []
        scales = []
        for name in ("k", "v"):
            pool = s[name].double()
            scale = None if case["fmt"] == "bf16" else 2.0 ** (s[name + "_scale"].double() - 127)
            x = s[name + "_new"].double()
            codes, steps = (x, None) if scale is None else _exact_codes(x)
            t = 0
            for b, (n, l) in enumerate(zip(s["new"], s["length"])):
                place = torch.arange(l - n, l)
                at, slot = table[b, place // page].long().cuda(), (place % page).cuda()
                pool[at, :, slot] = codes[t:t + n]
                if scale is not None:
                    scale[at, :, slot] = steps[t:t + n]
                t += n
            pools.append(pool)
            scales.append(scale)
        return (*pools, *scales)
    outs, lses = [], []
    t = 0
    for b, (n, l) in enumerate(zip(s["new"], s["length"])):
        k, v = context("k", b, 0, l), context("v", b, 0, l)
        q = s["q"][t:t + n].double().unflatten(1, (heads, group)).permute(1, 2, 0, 3)     # [heads, group, n, dim]
        row, col = torch.arange(l - n, l, device="cuda")[:, None], torch.arange(l, device="cuda")[None]
        hidden = (col > row) if not case["window"] else (col > row) | ((row - col >= case["window"]) & (col >= case["sinks"]))
        o, e = [], []
        for h in range(heads):
            z = (q[h] @ k[h].T) / dim ** 0.5
            z[:, hidden] = -torch.inf
            e.append(torch.logsumexp(z, -1))
            o.append(torch.exp(z - e[-1][..., None]) @ v[h])
        outs.append(torch.stack(o).permute(2, 0, 1, 3).flatten(1, 2))
        lses.append(torch.stack(e).permute(2, 0, 1).flatten(1))
        t += n
    return torch.cat(outs), torch.cat(lses)
