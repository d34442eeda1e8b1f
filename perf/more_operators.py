"""Cases of the operators of a decoder's 8-bit pass, with their plain forms.

Between the residual norm, the paged cache and the gate step a decoder multiplies, rotates and, at the
end, answers.  The operators here do that in the library's 8-bit format: the product of 8-bit
activations with 8-bit weights that have a scale per block of 128 x 128 (``linear``), the 8-bit
activations of a gated MLP (``quantise``), the norm of every query and key head with the position
rotation, into tensors or straight into the paged cache (``rotate``), and what a row of logits says of
a given token: its log probability and rank, the entropy, the top alternatives (``score``).

With ``own`` false, ``run`` is the plain form: elementary torch operations in 32 bits (angles in 64),
rounded once at the end.  With ``own`` true it calls the library's entry points.

8-bit values are e4m3 with one power-of-two scale per block (1 x 32, 1 x 128 or 128 x 128): the smallest
power for which no finite value of the block exceeds 448, kept between 2^-120 and 2^119 and stored as
its exponent plus 127.
"""
import random

import torch

own = False


# ----------------------------------------------------------------------------- cases
def listed():
    return [
        # one token through the query/key/value projection of a small Qwen-shaped model (1536 = 12 x 128, 2 cache heads): latency
        dict(name="linear_one_token", op="linear", T=1, N=2048, K=1536, block=128, out="bf16", bias=True),
        # one step of a full batch through the large Qwen-shaped model's projection (40 + 2 x 8 heads of 128), norm's output as it is
        dict(name="linear_step", op="linear", T=64, N=7168, K=5120, block=32, out="bf16", bias=True),
        # sequences that were just switched catch up: a ragged number of tokens, an odd number of features
        dict(name="linear_catch_up", op="linear", T=347, N=5000, K=4128, block=128, out="bf16", bias=False),
        # a prompt through the same projection: the compute-bound end
        dict(name="linear_prompt", op="linear", T=4099, N=7168, K=5120, block=128, out="bf16", bias=False),
        # logits of a batch from an 8-bit copy of the small Qwen-shaped model's head, kept in 32 bits for scoring
        dict(name="linear_head_f32", op="linear", T=61, N=152064, K=1536, block=32, out="f32", bias=False),
        # one step's gated MLP activations
        dict(name="quantise_step", op="quantise", rows=64, K=8960, block=128, gated=True),
        # a prompt's
        dict(name="quantise_prompt", op="quantise", rows=8191, K=13824, block=128, gated=True),
        # one step's queries, keys and values: norm, rotation, into the cache
        dict(name="rotate_step", op="rotate", form="write", fmt="bf16", B=64, new_lo=1, new_hi=1, len_lo=100, len_hi=9000,
             heads_q=40, heads_kv=8, dim=128, rot=128, interleaved=False, norm=True, page=16),
        # prompts into an 8-bit cache
        dict(name="rotate_prompts_e4m3", op="rotate", form="write", fmt="e4m3", B=12, new_lo=1100, new_hi=1900, len_lo=1900, len_hi=30001,
             heads_q=32, heads_kv=8, dim=128, rot=128, interleaved=False, norm=True, page=32),
        # tokens at far positions outside a cache, half of each head rotated, neighbouring pairs, no norm
        dict(name="rotate_dense", op="rotate", form="dense", fmt="bf16", B=1, new_lo=4001, new_hi=4001, len_lo=1000003, len_hi=1000003,
             heads_q=32, heads_kv=8, dim=64, rot=32, interleaved=True, norm=False, page=16),
        # the last token of one sequence scored, with five alternatives
        dict(name="score_one", op="score", rows=1, V=128256, out="f32", k=5, masked=0),
        # a prompt's tokens scored under the other model, twenty alternatives each; the vocabulary's padding is masked
        dict(name="score_prompt", op="score", rows=2041, V=152064, out="bf16", k=20, masked=399),
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
        op = rng.choice(["linear", "linear", "linear", "quantise", "rotate", "rotate", "score"])
        if op == "linear":
            c = dict(op=op, T=_log_int(rng, 1, 4099), N=_log_int(rng, 40, 152064), K=rng.choice([1536, 2048, 4096, 5120, 32 * rng.randint(2, 280)]),
                     block=rng.choice([32, 128]), out=rng.choice(["bf16", "bf16", "f32"]), bias=rng.random() < 0.5)
            if c["T"] * c["N"] > 40_000_000 or c["N"] * c["K"] > 250_000_000:
                continue
        elif op == "quantise":
            c = dict(op=op, rows=_log_int(rng, 1, 8191), K=rng.choice([1536, 2048, 4096, 5120, 8960, 13824, 32 * rng.randint(2, 432)]),
                     block=rng.choice([32, 128]), gated=rng.random() < 0.7)
        elif op == "rotate":
            heads_q, heads_kv, dim = rng.choice([(32, 8, 64), (32, 8, 128), (40, 8, 128), (12, 2, 128), (28, 4, 128), (16, 16, 64), (5, 1, 128)])
            B, new_hi = _log_int(rng, 1, 64), _log_int(rng, 1, 2600)
            len_hi = max(new_hi, _log_int(rng, 40, 32001))
            c = dict(op=op, form=rng.choice(["write", "write", "dense"]), fmt="bf16", B=B, new_lo=rng.randint(max(1, new_hi // 3), new_hi),
                     new_hi=new_hi, len_lo=rng.randint(max(new_hi, len_hi // 4), len_hi), len_hi=len_hi, heads_q=heads_q, heads_kv=heads_kv,
                     dim=dim, rot=rng.choice([dim, dim, dim // 2, 16]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.7,
                     page=rng.choice([16, 32, 64, 128]))
            if c["form"] == "write":
                c["fmt"] = rng.choice(["bf16", "e4m3"])
            if B * len_hi > 400_000:                                     # keeps the cache of a case within a GB or two
                continue
        else:
            c = dict(op=op, rows=_log_int(rng, 1, 2041), V=rng.choice([128256, 152064, _log_int(rng, 300, 160000)]),
                     out=rng.choice(["bf16", "f32", "f16"]), k=rng.choice([0, 1, 5, 8, 20, 64]), masked=rng.choice([0, 0, 64, 200]))
        w = work(c)
        if w["bytes"] <= top[op]["bytes"] and w["flops"] <= top[op]["flops"]:
            return c


def _lengths(case):
    """New tokens and context length (the new ones included) of every sequence; by the case alone."""
    spread = lambda step, at, b: (b * step + at) % 1.0                   # noqa: E731
    between = lambda lo, hi, u: lo + int(u * (hi - lo + 1))              # noqa: E731
    rows = range(case["B"])
    new = [between(case["new_lo"], case["new_hi"], spread(0.7548776662, 0.11, b)) for b in rows]
    return new, [max(new[b], between(case["len_lo"], case["len_hi"], spread(0.6180339887, 0.37, b))) for b in rows]


_SIZE = dict(bf16=2, f16=2, f32=4)
_TYPE = dict(bf16=torch.bfloat16, f16=torch.float16, f32=torch.float32)


def _up(n, m):
    return -(-n // m)


def work(case):
    op = case["op"]
    if op == "linear":
        T, N, K = case["T"], case["N"], case["K"]
        scales = T * _up(K, case["block"]) + _up(N, 128) * _up(K, 128)
        return {"bytes": (T + N) * K + scales + _SIZE[case["out"]] * T * N + (2 * N if case["bias"] else 0), "flops": 2 * T * N * K}
    if op == "quantise":
        n, K = case["rows"], case["K"]
        return {"bytes": n * ((4 if case["gated"] else 2) * K + K + _up(K, case["block"])), "flops": (6 if case["gated"] else 2) * n * K}
    if op == "score":
        n, V = case["rows"], case["V"]
        return {"bytes": n * (_SIZE[case["out"]] * V + 4 + 12 + 8 * min(case["k"], V)), "flops": 6 * n * V}
    n, dim = sum(_lengths(case)[0]), case["dim"]
    q, kv = case["heads_q"] * dim, case["heads_kv"] * dim
    bytes_ = n * 2 * 2 * q                                               # queries in and out
    if case["form"] == "dense":
        bytes_ += n * 2 * 2 * kv                                         # keys in and out
    else:
        bytes_ += n * 2 * (2 * kv + (2 * kv if case["fmt"] == "bf16" else kv + kv // 32))
    return {"bytes": bytes_, "flops": 8 * n * (q + kv)}


# ----------------------------------------------------------------------------- inputs
def _scale_bytes(amax):
    """Stored exponents of the scales for blocks of the given largest magnitudes (32-bit floats)."""
    mant, exp = torch.frexp(amax)                                       # amax = mant * 2^exp, 0.5 <= mant < 1
    k = torch.where(mant > 0.875, exp - 8, exp - 9)                     # 448 = 0.875 * 2^9
    k = torch.where(amax > 0, k.clamp(-120, 119), -120)
    return (k + 127).to(torch.uint8)


def _power(e):
    """2^e for whole numbers -126 .. 127, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x, block, block_rows=1):
    """[rows, n] values -> (e4m3 codes, stored scale exponents [rows / block_rows, n / block], both rounded up)."""
    rows, n = x.shape
    g = torch.nn.functional.pad(x, (0, -n % block, 0, -rows % block_rows))
    g = g.unflatten(1, (-1, block)).unflatten(0, (-1, block_rows))      # [row blocks, block_rows, blocks, block]
    stored = _scale_bytes(g.abs().amax((1, 3)))
    codes = (g * _power(127 - stored[:, None, :, None].int())).to(torch.float8_e4m3fn)
    return codes.flatten(2).flatten(0, 1)[:rows, :n].contiguous(), stored


def _values(codes, stored, block, block_rows=1):
    """32-bit values of codes [rows, n] with a scale per block_rows x block."""
    rows, n = codes.shape
    return codes.float() * _power(stored.int() - 127).repeat_interleave(block_rows, 0)[:rows].repeat_interleave(block, 1)[:, :n]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)   # noqa: E731
    s = dict(case=case)
    return dict(linear=_prepare_linear, quantise=_prepare_quantise, rotate=_prepare_rotate, score=_prepare_score)[case["op"]](s, case, seed, gen, rnd)


def _prepare_linear(s, case, seed, gen, rnd):
    T, N, K = case["T"], case["N"], case["K"]
    channel = torch.exp(0.7 * rnd(K))                                    # a few channels carry most of a normalised row
    s["x"], s["x_scale"] = _quantise(rnd(T, K) * channel, case["block"])
    s["w"] = torch.empty(N, K, dtype=torch.float8_e4m3fn, device="cuda")
    s["w_scale"] = torch.empty(_up(N, 128), _up(K, 128), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // (128 * K)) * 128
    for i in range(0, N, step):
        rows = min(step, N - i)
        spread = torch.exp2(0.5 * rnd(_up(rows, 128))).repeat_interleave(128)[:rows, None]      # row blocks of different size
        s["w"][i:i + rows], s["w_scale"][i // 128:_up(i + rows, 128)] = _quantise(rnd(rows, K) * spread * K ** -0.5, 128, 128)
    s["bias"] = (0.5 * rnd(N)).bfloat16() if case["bias"] else None
    s["out"] = torch.empty(T, N, dtype=_TYPE[case["out"]], device="cuda")
    s["workspace"] = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    return s


def _prepare_quantise(s, case, seed, gen, rnd):
    n, K = case["rows"], case["K"]
    channel = torch.exp(0.5 * rnd(K))
    if case["gated"]:                                                    # one projection's two halves, as the MLP makes them
        both = torch.empty(n, 2 * K, dtype=torch.bfloat16, device="cuda")
        both[:, :K], both[:, K:] = 2.0 * rnd(n, K), rnd(n, K) * channel
        s["gate"], s["x"] = both[:, :K], both[:, K:]
    else:
        s["gate"], s["x"] = None, (rnd(n, K) * channel).bfloat16()
    s["out"] = torch.empty(n, K, dtype=torch.float8_e4m3fn, device="cuda")
    s["out_scale"] = torch.empty(n, _up(K, case["block"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_rotate(s, case, seed, gen, rnd):
    B, heads, dim, page = case["B"], case["heads_kv"], case["dim"], case["page"]
    new, length = _lengths(case)
    n = sum(new)
    starts = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32)
    s.update(new=new, length=length, total=n, new_start=starts.cuda(), kv_len=torch.tensor(length, dtype=torch.int32).cuda(),
             status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    qkv = torch.empty(n, case["heads_q"] + 2 * heads, dim, dtype=torch.bfloat16, device="cuda")      # one projection, used in slices
    channel = torch.exp(0.5 * rnd(dim))
    qkv.copy_(rnd(*qkv.shape) * channel)
    s["q"], s["k"], s["v"] = qkv[:, :case["heads_q"]], qkv[:, case["heads_q"]:case["heads_q"] + heads], qkv[:, case["heads_q"] + heads:]
    s["q_weight"] = (1.0 + 0.2 * rnd(dim)).bfloat16() if case["norm"] else None
    s["k_weight"] = (1.0 + 0.2 * rnd(dim)).bfloat16() if case["norm"] else None
    s["inv_freq"] = (500000.0 ** -(torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])).float().cuda()
    s["q_out"] = torch.empty(n, case["heads_q"], dim, dtype=torch.bfloat16, device="cuda")
    if case["form"] == "dense":
        s["k_out"] = torch.empty(n, heads, dim, dtype=torch.bfloat16, device="cuda")
        b, i = _owners(s)
        s["positions"] = ((s["kv_len"] - s["new_start"].diff())[b] + i).to(torch.int32)
        return s
    pages = [_up(l, page) for l in length]
    n_pages, width = sum(pages) + 3, max(pages)
    order = list(range(n_pages))
    random.Random(seed).shuffle(order)                                   # pages in no order, as a pool hands them out
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = torch.tensor(order[at:at + pages[b]], dtype=torch.int32)
        at += pages[b]
    s.update(table=table.cuda(), max_new=max(new), max_len=max(length))
    for name in ("k", "v"):                                              # what earlier steps left there is not read
        s[name + "_pool"] = torch.zeros(n_pages, heads, page, dim, dtype=torch.bfloat16 if case["fmt"] == "bf16" else torch.float8_e4m3fn, device="cuda")
        s[name + "_scale"] = None if case["fmt"] == "bf16" else torch.zeros(n_pages, heads, page, dim // 32, dtype=torch.uint8, device="cuda")
    return s


def _prepare_score(s, case, seed, gen, rnd):
    n, V = case["rows"], case["V"]
    real = V - case["masked"]
    s["logits"] = torch.empty(n, V, dtype=_TYPE[case["out"]], device="cuda")
    step = max(1, (1 << 26) // V)
    likely = torch.randint(0, real, (n, 32), device="cuda", generator=gen)     # the few words that fit, some much better than others
    for i in range(0, n, step):
        z = 2.0 * rnd(min(step, n - i), V)
        z.scatter_add_(1, likely[i:i + step], 4.0 + 3.0 * rnd(z.shape[0], 32))
        z[:, real:] = float("-inf")
        s["logits"][i:i + step] = z
    other = torch.randint(0, real, (n,), device="cuda", generator=gen)
    s["tokens"] = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.8, likely[:, 0], other).int()
    s["logprob"], s["entropy"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    s["rank"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["top"] = torch.empty(n, case["k"], dtype=torch.int32, device="cuda")
    s["top_logprob"] = torch.empty(n, case["k"], device="cuda")
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["workspace"] = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    return s


# ----------------------------------------------------------------------------- one pass
def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


def _e8m0(stored):
    return None if stored is None else stored.view(torch.float8_e8m0fnu)


def _own(s):
    from paper_2502_06833_b200 import binding as E
    case, stream = s["case"], E.current_stream()
    if case["op"] == "linear":
        if "x_matrix" not in s:                                          # a program describes its weights and buffers once
            s["x_matrix"] = E.ead_e4m3_matrix(s["x"], s["x_scale"], block=(1, case["block"]))
            s["w_matrix"] = E.ead_e4m3_matrix(s["w"], s["w_scale"], block=(128, 128))
        E.ead_linear(s["x_matrix"], s["w_matrix"], s["out"], bias=s["bias"], stream=stream)
        return s["out"]
    if case["op"] == "quantise":
        if "matrix" not in s:
            s["matrix"] = E.ead_e4m3_matrix(s["out"], s["out_scale"], block=(1, case["block"]))
        E.ead_quantise(s["x"], s["matrix"], gate=s["gate"], stream=stream)
        return s["out"], _e8m0(s["out_scale"])
    if case["op"] == "score":
        E.ead_token_logprobs(s["logits"], s["tokens"], logprob=s["logprob"], entropy=s["entropy"], rank=s["rank"], top=s["top"],
                             top_logprob=s["top_logprob"], workspace=s["workspace"], status=s["status"], stream=stream)
        return s["logprob"], s["entropy"], s["rank"], s["top"], s["top_logprob"]
    if "rope" not in s:
        s["rope"] = E.ead_rope(s["inv_freq"], case["dim"], interleaved=case["interleaved"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6)
        if case["form"] == "write":
            s["cache"] = E.ead_kv_cache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
            s["batch"] = E.ead_kv_batch(s["table"], s["new_start"], s["kv_len"], n_tokens=s["total"], max_new=s["max_new"], max_len=s["max_len"])
    if case["form"] == "dense":
        E.ead_qk_norm_rope(s["rope"], s["positions"], s["q"], s["k"], s["q_out"], s["k_out"], stream=stream)
        return s["q_out"], s["k_out"]
    E.ead_kv_rotate_write(s["rope"], s["cache"], s["batch"], s["q"], s["k"], s["v"], s["q_out"], status=s["status"], stream=stream)
    return s["q_out"], s["k_pool"], s["v_pool"], _e8m0(s["k_scale"]), _e8m0(s["v_scale"])


def _plain_linear(s):
    out = _values(s["x"], s["x_scale"], s["case"]["block"]) @ _values(s["w"], s["w_scale"], 128, 128).T
    if s["bias"] is not None:
        out += s["bias"].float()
    return out.to(s["out"].dtype)


def _plain_quantise(s):
    y = s["x"].float()
    if s["gate"] is not None:
        g = s["gate"].float()
        y = g / (1.0 + torch.exp(-g)) * y
    codes, stored = _quantise(y, s["case"]["block"])
    return codes, _e8m0(stored)


def _owners(s):
    """Sequence and index within the sequence's new tokens, for every new token of the step."""
    at = torch.arange(s["total"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["new_start"][1:], at, right=True)
    return b, at - s["new_start"][b]


def _rotated(x, weight, place, s):
    case, half = s["case"], s["case"]["rot"] // 2
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight.float()
    angle = place.double()[:, None, None] * s["inv_freq"].double()
    c, d = angle.cos().float(), angle.sin().float()
    a, b = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if case["interleaved"] else (y[..., :half], y[..., half:2 * half])
    turned = torch.stack((a * c - b * d, b * c + a * d), -1 if case["interleaved"] else -2).flatten(-2)
    return torch.cat((turned, y[..., 2 * half:]), -1)


def _put(pool, scale, new, at, slot):
    if scale is None:
        pool[at, :, slot] = new.to(pool.dtype)
    else:
        codes, stored = _quantise(new.reshape(-1, new.shape[-1]), 32)
        pool.view(torch.uint8)[at, :, slot] = codes.view(torch.uint8).view(new.shape)
        scale[at, :, slot] = stored.view(*new.shape[:-1], -1)


def _plain_rotate(s):
    case = s["case"]
    if case["form"] == "dense":
        place = s["positions"]
    else:
        b, i = _owners(s)
        place = (s["kv_len"] - s["new_start"].diff())[b] + i
    q, k = _rotated(s["q"], s["q_weight"], place, s).to(torch.bfloat16), _rotated(s["k"], s["k_weight"], place, s)
    if case["form"] == "dense":
        return q, k.to(torch.bfloat16)
    at, slot = s["table"][b, place // case["page"]].long(), (place % case["page"]).long()
    _put(s["k_pool"], s["k_scale"], k, at, slot)
    _put(s["v_pool"], s["v_scale"], s["v"].float(), at, slot)
    return q, s["k_pool"], s["v_pool"], _e8m0(s["k_scale"]), _e8m0(s["v_scale"])


def _plain_score(s):
    V, k, token = s["case"]["V"], s["case"]["k"], s["tokens"].long()[:, None]
    z = s["logits"].float()
    index = torch.arange(V, device="cuda")
    given = z.gather(1, token)
    rank = ((z > given) | ((z == given) & (index < token))).sum(1)       # how many come before it
    bits = z.view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7fffffff), bits) * (1 << 32) + (V - 1 - index)      # ties go to the lowest index
    best = V - 1 - order.topk(min(k, V), 1).values % (1 << 32)
    del bits, order
    best_z = z.gather(1, best)
    top = z.amax(1, keepdim=True)
    d = z.sub_(top)
    p = d.exp()
    total = p.sum(1, keepdim=True)
    log_total = total.log()
    entropy = log_total - torch.where(p > 0, p * d, 0.0).sum(1, keepdim=True) / total
    return ((given - top - log_total).squeeze(1), entropy.squeeze(1), rank.int(), best.int(), best_z - top - log_total)


_PLAIN = dict(linear=_plain_linear, quantise=_plain_quantise, rotate=_plain_rotate, score=_plain_score)


# ----------------------------------------------------------------------------- in 64 bits
def _two(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_codes(x, block):
    """Block scales and e4m3 values of 64-bit numbers, by logarithms corrected to the definition, and a rounding grid."""
    n = x.shape[-1]
    width = _up(n, block) * block
    g = torch.cat((x, x.new_zeros(*x.shape[:-1], width - n)), -1).unflatten(-1, (-1, block))
    amax = g.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(amax.clamp_min(2.0 ** -140) / 448.0)).clamp(-120, 119)
    k = torch.where(amax > 448.0 * _two(k), k + 1, torch.where(amax <= 448.0 * _two(k - 1), k - 1, k)).clamp(-120, 119)
    z = g / _two(k)
    step = _two(torch.frexp(z.abs().clamp_min(2.0 ** -6)).exponent - 4)      # spacing of e4m3 at each magnitude
    return (torch.round(z / step) * step).flatten(-2)[..., :n].contiguous(), _two(k).squeeze(-1)     # round() takes ties to even


def exact(case, seed):
    return dict(linear=_exact_linear, quantise=_exact_quantise, rotate=_exact_rotate, score=_exact_score)[case["op"]](case, prepare(case, seed))


def _exact_linear(case, s):
    T, N, K, block = case["T"], case["N"], case["K"], case["block"]
    x, out = s["x"].double(), torch.empty(T, N, dtype=torch.float64, device="cuda")
    for j in range(_up(K, block)):
        x[:, j * block:(j + 1) * block] *= _two(s["x_scale"][:, j:j + 1].long() - 127)
    wide = 128 * 64                                                      # features at a time
    for i in range(0, N, wide):
        w = s["w"][i:i + wide].double()
        for j in range(_up(K, 128)):
            step = _two(s["w_scale"][i // 128:i // 128 + 64, j].long() - 127)
            w[:, j * 128:(j + 1) * 128] *= step.repeat_interleave(128)[:w.shape[0], None]
        out[:, i:i + wide] = x @ w.T
    return out if s["bias"] is None else out + s["bias"].double()


def _exact_quantise(case, s):
    codes, steps = [], []
    for x, g in zip(s["x"].split(1024), s["gate"].split(1024) if case["gated"] else [None] * _up(case["rows"], 1024)):
        y = x.double()
        if g is not None:
            y = y * g.double() * torch.sigmoid(g.double())
        c, k = _exact_codes(y, case["block"])
        codes.append(c)
        steps.append(k)
    return torch.cat(codes), torch.cat(steps)


def _exact_rotate(case, s):
    dim, half = case["dim"], case["rot"] // 2
    pair = torch.arange(half, device="cuda")
    first, second = (2 * pair, 2 * pair + 1) if case["interleaved"] else (pair, pair + half)
    place = torch.cat([torch.arange(l - n, l) for n, l in zip(s["new"], s["length"])]).cuda()

    def turn(x, weight):
        y = x.double()
        if weight is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / dim + 1e-6) * weight.double()
        spin = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), place.double()[:, None] * s["inv_freq"].double())[:, None]
        z = torch.complex(y[..., first], y[..., second]) * spin
        y[..., first], y[..., second] = z.real, z.imag
        return y

    q, k = turn(s["q"], s["q_weight"]), turn(s["k"], s["k_weight"])
    if case["form"] == "dense":
        return q, k
    table, page = s["table"].cpu(), case["page"]
    pools, scales = [], []
    for name, x in (("k", k), ("v", s["v"].double())):
        pool = s[name + "_pool"].double()
        scale = None if case["fmt"] == "bf16" else _two(s[name + "_scale"].long() - 127)
        codes, steps = (x, None) if scale is None else _exact_codes(x, 32)
        t = 0
        for b, (n, l) in enumerate(zip(s["new"], s["length"])):
            p = torch.arange(l - n, l)
            at, slot = table[b, p // page].long().cuda(), (p % page).cuda()
            pool[at, :, slot] = codes[t:t + n]
            if scale is not None:
                scale[at, :, slot] = steps[t:t + n]
            t += n
        pools.append(pool)
        scales.append(scale)
    return (q, *pools, *scales)


def _exact_score(case, s):
    outs = []
    for z, token in zip(s["logits"].split(256), s["tokens"].long().split(256)):
        z = z.double()
        lse = torch.logsumexp(z, 1, keepdim=True)
        order = torch.sort(z, dim=1, descending=True, stable=True).indices
        logp = z - lse
        entropy = -(torch.nan_to_num(logp, neginf=0.0) * logp.exp()).sum(1)
        outs.append((logp.gather(1, token[:, None])[:, 0], entropy, (order == token[:, None]).int().argmax(1).int(),
                     order[:, :case["k"]].int(), logp.gather(1, order[:, :case["k"]])))
    return tuple(torch.cat(o) for o in zip(*outs))
