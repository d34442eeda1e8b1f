"""The operators of a decoder's 8-bit pass run one after the other as a decoder layer uses them: every one is checked in 64 bits on what
the one before it really gave, so that errors do not add up.  And the example with them."""
import os
import sys

import numpy as np
import pytest
import torch

import pass_util as P
from decoder_util import Context

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def E():
    from paper_2502_06833_b200 import binding
    return binding


def _matrix(E, rows, cols, block):
    return E.ead_e4m3_matrix(torch.empty(rows, cols, dtype=torch.uint8, device="cuda"),
                             torch.empty(P.up(rows, block[0]), P.up(cols, block[1]), dtype=torch.uint8, device="cuda"), block=block)


def _values(m):
    return P.values(m.held[0].cpu().numpy(), m.held[1].cpu().numpy(), m.block_cols, m.block_rows)


def _check_product(out, x, w, bias=None):
    xv, wv = _values(x), _values(w)
    want, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    if bias is not None:
        want = want + bias.double().cpu().numpy()
        size = size + np.abs(bias.double().cpu().numpy())
    tol = (x.cols / 32 + 16) * 2.0 ** -23 * size                         # 32-bit sums, K / 32 of them, and the join of parts
    tol += torch.finfo(out.dtype).eps / 2 * (np.abs(want) + tol)
    d = np.abs(out.double().cpu().numpy() - want)
    assert (d <= tol).all(), (d / tol).max()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,length", [([1, 1, 1], [1, 40, 333]), ([5, 70, 1, 200], [5, 200, 17, 200])])
def test_a_layer_in_8_bits(E, fmt, new, length):
    hidden, hq, hk, dim, inner, V = 512, 8, 2, 64, 768, 1000
    g = torch.Generator().manual_seed(len(new))
    rnd = lambda *s: torch.randn(*s, generator=g)                        # noqa: E731
    n, stream, status = sum(new), E.current_stream(), torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx = Context(new, length, hk, dim, 16, fmt, seed=3)                 # earlier tokens are in the cache
    weights = {}
    for name, rows, cols in (("qkv", (hq + 2 * hk) * dim, hidden), ("out", hidden, hq * dim), ("up", 2 * inner, hidden), ("down", hidden, inner), ("head", V, hidden)):
        weights[name] = _matrix(E, rows, cols, (128, 128))
        w = (rnd(rows, cols) * cols ** -0.5).bfloat16()
        E.ead_quantise(w.cuda(), weights[name], stream=stream)
        codes, scale = P.quantise(w.double().numpy(), 128, 128)
        assert np.array_equal(weights[name].held[0].cpu().numpy(), codes) and np.array_equal(weights[name].held[1].cpu().numpy(), scale)
    x, res = (2 * rnd(n, hidden)).bfloat16().cuda(), rnd(n, hidden).bfloat16().cuda()
    ones = (1 + 0.1 * rnd(hidden)).bfloat16().cuda()

    def norm(add, residual):
        """8-bit rows of the norm; the values behind them are checked elsewhere."""
        m = _matrix(E, n, hidden, (1, 32))
        E.ead_add_rmsnorm(add, ones, m.held[0], residual=residual, residual_out=residual, out_scale=m.held[1], stream=stream)
        return m

    def product(x, name, dtype=torch.bfloat16, bias=None):
        out = torch.empty(n, weights[name].rows, dtype=dtype, device="cuda")
        E.ead_linear(x, weights[name], out, bias=bias, status=status, stream=stream)
        _check_product(out, x, weights[name], bias)
        return out

    bias = rnd((hq + 2 * hk) * dim).bfloat16().cuda()
    qkv = product(norm(x, res), "qkv", bias=bias).view(n, hq + 2 * hk, dim)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    f = (10000.0 ** -(torch.arange(0, dim, 2, dtype=torch.float64) / dim)).float()
    qw, kw = (1 + 0.2 * rnd(dim)).bfloat16(), (1 + 0.2 * rnd(dim)).bfloat16()
    rope = E.ead_rope(f.cuda(), dim, q_weight=qw.cuda(), k_weight=kw.cuda())
    place = torch.cat([torch.arange(l - m, l) for m, l in zip(new, length)])
    want_q, size_q = P.rotated(q.cpu(), qw, place, f, False, 1e-6)
    want_k, size_k = P.rotated(k.cpu(), kw, place, f, False, 1e-6)
    cache, batch = ctx.cache(E), ctx.batch(E)
    E.ead_kv_rotate_write(rope, cache, batch, q, k, v, q, status=status, stream=stream)
    tol = lambda w, s: 2.0 ** -19 * s + 2.0 ** -8 * (w.abs() + 2.0 ** -19 * s)       # noqa: E731  (as where the operator is tested by itself)
    assert ((q.cpu().double() - want_q).abs() <= tol(want_q, size_q)).all()
    # what attention sees: the cache's own values, read back
    every = sum(length)
    starts = torch.tensor([0] + list(length), dtype=torch.int32).cumsum(0).int().cuda()
    kk, vv = (torch.empty(every, hk, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    E.ead_kv_read(cache, E.ead_kv_batch(ctx.d_table, starts, n_tokens=every, max_new=max(length), max_len=max(length)), kk, vv, status=status, stream=stream)
    at = torch.cat([torch.arange(l - m, l) + s for m, l, s in zip(new, length, np.cumsum([0] + list(length)))])
    near = (kk[at.cuda()].cpu().double() - want_k).abs()
    assert (near <= (tol(want_k, size_k) if fmt == "bf16" else 2.0 ** -4 * want_k.abs().amax(-1, keepdim=True) + tol(want_k, size_k))).all()
    out = torch.empty(n, hq, dim, dtype=torch.bfloat16, device="cuda")
    space = torch.zeros(E.EAD_KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    E.ead_kv_attention(cache, batch, q, out, scale=dim ** -0.5, workspace=space, status=status, stream=stream)
    from decoder_util import attention
    o = 0
    for b, l in enumerate(length):
        ctx.host["k"][b], ctx.host["v"][b] = kk[o:o + l].cpu().double(), vv[o:o + l].cpu().double()
        o += l
    w_out, _, tol_o, _ = attention(ctx, q.cpu(), dim ** -0.5, 0, 0)
    assert ((out.cpu().double() - w_out).abs() <= tol_o).all()

    def quantised(y, gate=None):
        m = _matrix(E, n, y.shape[1], (1, 128))
        E.ead_quantise(y, m, gate=gate, stream=stream)
        want = y.double().cpu().numpy()
        if gate is not None:
            a = gate.double().cpu().numpy()
            want = want * a / (1 + np.exp(-a))
        top = np.repeat(np.maximum.reduceat(np.abs(want), np.arange(0, want.shape[1], 128), 1), 128, 1)[:, :want.shape[1]]
        assert (np.abs(_values(m) - want) <= 2.0 ** -4 * 1.01 * np.abs(want) + 2.0 ** -17 * top).all()     # half a step, or half of the smallest (2^-10 of the scale, 2^-17 of the largest value)
        return m

    y = product(quantised(out.view(n, -1)), "out")
    gate, up = product(norm(y, res), "up").chunk(2, -1)
    y = product(quantised(up, gate), "down")
    logits = product(norm(y, res), "head", torch.float32)
    tokens = torch.randint(0, V, (n,), generator=g)
    lp, h = (torch.empty(n, device="cuda") for _ in range(2))
    rank, top, top_lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, 5, dtype=torch.int32, device="cuda"), torch.empty(n, 5, device="cuda")
    E.ead_token_logprobs(logits, tokens.int().cuda(), logprob=lp, entropy=h, rank=rank, top=top, top_logprob=top_lp,
                         workspace=torch.zeros(E.EAD_LOGPROB_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda"), status=status, stream=stream)
    w_lp, w_h, w_rank, w_top, w_top_lp = P.scores(logits.cpu().double(), tokens, 5)
    room = 2.0 ** -20 * (1 + 16 + logits.abs().max().item())
    assert torch.equal(rank.cpu().long(), w_rank) and torch.equal(top.cpu().long(), w_top)
    assert ((lp.cpu().double() - w_lp).abs() <= room).all() and ((h.cpu().double() - w_h).abs() <= room).all() and ((top_lp.cpu().double() - w_top_lp).abs() <= room).all()
    assert status.item() == 0


def test_example_with_rotation_catches_up():
    """As without rotation; a query's and a key's rounding more per layer."""
    import adaptive_pair as A
    history, log, small, large = A.generate(steps=30, rope=True)
    flat = sum(log, [])
    assert 0 < sum(flat) < len(flat)
    everyone = set(range(len(history)))
    for m in (small, large):
        late = m.step(history, everyone).float()
        m.forget()
        whole = m.step(history, everyone).float()
        assert m.status.item() == 0
        err = (late - whole).square().mean().sqrt() / whole.square().mean().sqrt()
        assert err < 18 * 2.0 ** -8, err


@pytest.mark.parametrize("kw", [dict(w8=True), dict(w8=True, rope=True, e4m3=True), dict(rope=True), dict()])
def test_example_scores_what_it_produced(kw):
    import adaptive_pair as A
    history, log, small, large = A.generate(steps=20, **kw)
    for m in (small, large):
        got = m.score(history)
        assert m.status.item() == 0
        for b, h in enumerate(history):
            assert len(got["logprob"][b]) == len(got["rank"][b]) == len(got["entropy"][b]) == len(h) - 1
            lp, rank, entropy = (torch.tensor(got[k][b]) for k in ("logprob", "rank", "entropy"))
            assert (lp < 0).all() and lp.isfinite().all() and (entropy > 0).all() and (entropy <= np.log(512) + 1e-4).all()
            assert (rank >= 0).all() and (rank < 512).all()
            assert (lp <= -torch.log1p(rank.float()) + 1e-4).all()       # rank tokens are at least as likely: p <= 1 / (rank + 1)


@pytest.mark.parametrize("T", [3, 200])
def test_calls_back_to_back_equal_calls_one_at_a_time(E, T):
    """A kernel's setup runs under the end of the one before it; what that one writes must be what it reads.  Every round has other numbers in the same
    buffers; once with a wait after every call, once without any."""
    K, V, rounds = 640, 3000, 25
    g = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()              # noqa: E731
    xs, gates = [rnd(T, K) for _ in range(rounds)], [rnd(T, K) for _ in range(rounds)]
    w = _matrix(E, V, K, (128, 128))
    E.ead_quantise(rnd(V, K), w, stream=E.current_stream())
    tokens = [torch.randint(0, V, (T,), generator=g, device="cuda").int() for _ in range(rounds)]
    x, gate, token = torch.empty_like(xs[0]), torch.empty_like(xs[0]), torch.empty_like(tokens[0])
    q, logits, space = _matrix(E, T, K, (1, 128)), torch.empty(T, V, device="cuda"), torch.zeros(E.EAD_LOGPROB_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    f = (10000.0 ** -(torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().cuda()
    rope, place = E.ead_rope(f, 64), torch.arange(T, dtype=torch.int32, device="cuda")

    def go(wait):
        out = []
        for i in range(rounds):
            x.copy_(xs[i])
            gate.copy_(gates[i])
            token.copy_(tokens[i])
            heads = x.view(T, K // 64, 64)
            lp, rank, top = torch.empty(T, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda"), torch.empty(T, 4, dtype=torch.int32, device="cuda")
            s = E.current_stream()
            for call in (lambda: E.ead_qk_norm_rope(rope, place, heads, None, heads, None, stream=s), lambda: E.ead_quantise(x, q, gate=gate, stream=s),
                         lambda: E.ead_linear(q, w, logits, stream=s),
                         lambda: E.ead_token_logprobs(logits, token, logprob=lp, rank=rank, top=top, workspace=space, stream=s)):
                call()
                if wait:
                    torch.cuda.synchronize()
            out.append((x.clone(), logits.clone(), lp, rank, top))
        torch.cuda.synchronize()
        return out
    for a, b in zip(go(True), go(False)):
        assert all(torch.equal(p, r) for p, r in zip(a, b))
