"""The operators of a decoder's 8-bit pass at sizes where a block or warp goes round its loops many times: several tiles per pair of blocks, rings of
shared memory used again, rows that are not cut, more rows than a grid has.  Against plain 64-bit statements."""
import math

import numpy as np
import pytest
import torch

import pass_util as P
from decoder_util import Context, e4m3_grid
from test_gpu_pass_ops import DTYPES, Product, _check_rotated, _rope, _same_blocks

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    from paper_2502_06833_b200 import binding
    return binding


@pytest.fixture(scope="module")
def space(E):
    return torch.zeros(E.EAD_LOGPROB_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ----------------------------------------------------------------------------- product
def _product_limits(p, dtype):
    """Product.check's: K / 32 + 16 roundings of 2^-23 of the magnitudes, then half a step of the output."""
    x, w = torch.from_numpy(p.xv).cuda(), torch.from_numpy(p.wv).cuda()
    bias = p.bias.double()
    want, size = x @ w.T + bias, x.abs() @ w.abs().T + bias.abs()
    tol = (x.shape[1] / 32 + 16) * 2.0 ** -23 * size
    return want, tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol) + 1e-37


@pytest.mark.parametrize("block", [32, 128])
@pytest.mark.parametrize("T,N,K", [(1999, 7100, 1184), (700, 20011, 672), (3001, 3500, 2080), (150, 38500, 672), (33, 57001, 288)])
def test_linear_many_tiles(E, block, T, N, K):
    """Several tiles per pair of blocks (or single block), each with several groups of scales, the last ones cut short in features, tokens
    and K; and the same again."""
    p = Product(E, T, N, K, block, seed=T + block)
    for dtype in (torch.bfloat16, torch.float32):
        want, tol = _product_limits(p, dtype)
        first = p.run(E, dtype).cuda()
        d = (first.double() - want).abs()
        assert not d.isnan().any() and (d <= tol).all(), (d / tol).max()
        for _ in range(3):
            assert torch.equal(p.run(E, dtype).cuda(), first)


# ----------------------------------------------------------------------------- quantisation
def _scale_byte(amax):
    mant, exp = torch.frexp(amax)
    return torch.where(amax > 0, torch.where(mant > 0.875, exp - 8, exp - 9).clamp(-120, 119), -120) + 127      # 448 = 0.875 * 2^9


def _blocks_of(x, block):
    """Codes and scale bytes of bf16 rows by torch's conversion: a power of two changes no digit of a value that stays normal."""
    cols = x.shape[1]
    g = torch.nn.functional.pad(x.double(), (0, -cols % block)).unflatten(1, (-1, block))
    byte = _scale_byte(g.abs().amax(2))
    codes = (g * torch.exp2(127.0 - byte)[..., None]).float().to(torch.float8_e4m3fn)
    return codes.flatten(1)[:, :cols].view(torch.uint8), byte.to(torch.uint8)


@pytest.mark.parametrize("block", [32, 128])
@pytest.mark.parametrize("rows,cols", [(870, 16416), (4100, 16416), (9001, 3104)])
def test_quantise_rows_in_long_stretches(E, block, rows, cols):
    """A warp has 3, 14 and 6 passes of 512 values (or a few less): exactly the definition's codes."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g, device="cuda").float())).bfloat16()
    x[3, 512:1024] = 0
    codes = torch.full((rows, cols + 32), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(rows, P.up(cols, block), dtype=torch.uint8, device="cuda")
    E.ead_quantise(x, E.ead_e4m3_matrix(codes[:, :cols], scale, block=(1, block)))
    for r in range(0, rows, 500):
        want = _blocks_of(x[r:r + 500], block)
        assert torch.equal(scale[r:r + 500], want[1]) and torch.equal(codes[r:r + 500, :cols], want[0])
    assert (codes[:, cols:] == 0x55).all() and (scale[3, 512 // block:1024 // block] == 7).all()


def _gated_error(gate):
    """Relative error of a gated value: 2^-22 each for the exponential and the quotient by the special function unit, half a unit (2^-24) for the sum and the
    product, and the exponential's argument, gate times log2 e, is off by its rounding and the constant's: 1.22 x 2^-24 of the gate."""
    return 2.0 ** -20 + 1.25 * 2.0 ** -24 * gate.double().abs()


def _check_codes(codes, scale, y, tol, block):
    """Scales and codes are those of some value within tol of y (64 bits): no half step is given away beside it."""
    rows, cols = y.shape
    pad = lambda t: torch.nn.functional.pad(t, (0, -cols % block)).unflatten(1, (-1, block))     # noqa: E731
    low, high = _scale_byte(pad((y.abs() - tol).clamp_min(0)).amax(2)), _scale_byte(pad(y.abs() + tol).amax(2))
    byte = scale.long()
    assert ((byte >= low) & (byte <= high)).all()
    grid = torch.from_numpy(e4m3_grid()).cuda()
    between = (grid[1:] + grid[:-1]) / 2
    step = torch.exp2(byte.double() - 127).repeat_interleave(block, 1)[:, :cols]
    below = torch.bucketize(((y.abs() - tol) / step), between, right=False)            # on a border: the code below it, or above
    above = torch.bucketize(((y.abs() + tol) / step), between, right=True)
    size = (codes & 0x7F).long()
    wrong = (size < below) | (size > above) | ((size > 0) & ((codes >= 0x80) != (y < 0)))
    assert not wrong.any(), (int(wrong.sum()), y.numel())


def _gated(E, x, gate, block):
    rows, cols = x.shape
    codes = torch.zeros(rows, cols, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(rows, P.up(cols, block), dtype=torch.uint8, device="cuda")
    E.ead_quantise(x, E.ead_e4m3_matrix(codes, scale, block=(1, block)), gate=gate)
    y = x.double() * gate.double() / (1 + torch.exp(-gate.double()))
    _check_codes(codes, scale, y, _gated_error(gate) * y.abs() + 2.0 ** -125, block)


@pytest.mark.parametrize("block", [32, 128])
@pytest.mark.parametrize("rows,cols", [(900, 16416), (12, 96)])
def test_quantise_gated_in_long_stretches(E, block, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows)
    both = (3 * torch.randn(rows, 2, cols, generator=g, device="cuda")).bfloat16()
    _gated(E, both[:, 1], both[:, 0], block)


@pytest.mark.parametrize("block", [32, 128])
def test_quantise_every_gate(E, block):
    """Every gate of at most 87.25 above 2^-7, with every value of one octave: a block's values are what the gate makes of about 1."""
    bits = torch.arange(0x3C00, 0x42AF, dtype=torch.int32, device="cuda")                        # 2^-7 .. 87.0
    gate = torch.cat((bits, bits | 0x8000)).to(torch.int16).view(torch.bfloat16)[:, None].expand(-1, 128).contiguous()
    octave = torch.arange(0x3F80, 0x4000, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16)
    lift = torch.exp2(torch.floor(-gate[:, :1].float() / math.log(2)).clamp(-6, 120))
    _gated(E, (octave.float() * lift).bfloat16(), gate, block)


# ----------------------------------------------------------------------------- norm and rotation
# 2400 tokens are more than the warps that a call of few tokens is divided into: a warp has a token's 10 to 12 runs.
ROPES = [(128, 128, False, (1, 1), 32, 8), (128, 128, False, (1, 0), 30, 7), (64, 64, False, (0, 1), 60, 16), (64, 32, True, (0, 0), 32, 8), (128, 48, False, (1, 0), 21, 3),
         (128, 128, True, (0, 1), 16, 4), (64, 0, False, (1, 1), 40, 5)]


@pytest.mark.parametrize("dim,rot,interleaved,norm,hq,hk", ROPES)
def test_qk_norm_rope_many_tokens(E, dim, rot, interleaved, norm, hq, hk):
    n = 2400
    g = torch.Generator().manual_seed(hq)
    rope, f, w = _rope(E, dim, rot, interleaved, norm, hq)
    place = torch.randint(0, 100000, (n,), generator=g).int()
    both = (torch.randn(n, hq + hk, dim, generator=g) * torch.exp(torch.randn(dim, generator=g))).bfloat16()
    dev = both.cuda()
    out = torch.full((n, hq + hk + 1, dim), -7.0, dtype=torch.bfloat16, device="cuda")
    E.ead_qk_norm_rope(rope, place.cuda(), dev[:, :hq], dev[:, hq:], out[:, :hq], out[:, hq:hq + hk])
    assert (out[:, hq + hk:] == -7.0).all()
    _check_rotated(out[:, :hq].cpu(), *P.rotated(both[:, :hq], w[0], place, f, interleaved, 1e-5))
    _check_rotated(out[:, hq:hq + hk].cpu(), *P.rotated(both[:, hq:], w[1], place, f, interleaved, 1e-5))
    E.ead_qk_norm_rope(rope, place.cuda(), dev[:, :hq], dev[:, hq:], dev[:, :hq], dev[:, hq:])
    assert torch.equal(dev, out[:, :hq + hk])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim,rot,interleaved,norm,hq,heads", ROPES)
def test_kv_rotate_write_prompts(E, fmt, dim, rot, interleaved, norm, hq, heads):
    """As for ragged steps: queries, keys (normalised and not) and values of prompts; what the cache held elsewhere stays."""
    new, length, page = [1190, 0, 1, 1209], [1190, 40, 700, 1500], 16
    ctx = Context(new, length, heads, dim, page, fmt, seed=hq, stale=0.25)
    n = sum(new)
    g = torch.Generator().manual_seed(hq)
    both = (torch.randn(n, hq + 2 * heads, dim, generator=g) * torch.exp(0.5 * torch.randn(dim, generator=g))).bfloat16()
    dev = both.cuda()
    rope, f, w = _rope(E, dim, rot, interleaved, norm, 3)
    place = torch.cat([torch.arange(l - m, l) for m, l in zip(new, length)]).int()
    before = {s: t.clone() for s, t in ctx.dev.items()}
    out, st = torch.zeros(n, hq, dim, dtype=torch.bfloat16, device="cuda"), _status()
    E.ead_kv_rotate_write(rope, ctx.cache(E), ctx.batch(E), dev[:, :hq], dev[:, hq:hq + heads], dev[:, hq + heads:], out, status=st)
    assert st.item() == 0
    _check_rotated(out.cpu(), *P.rotated(both[:, :hq], w[0], place, f, interleaved, 1e-5))
    owner = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new))
    pages, slots = torch.from_numpy(ctx.table)[owner, place.long() // page].long(), place.long() % page
    k_want, k_size = P.rotated(both[:, hq:hq + heads], w[1], place, f, interleaved, 1e-5)
    v_want = both[:, hq + heads:].double()
    flat = lambda t: t.reshape(-1, t.shape[-1]).numpy()                  # noqa: E731
    same = lambda a, b: torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))   # noqa: E731
    for name, want, tol in (("k", k_want, 2.0 ** -19 * k_size), ("v", v_want, torch.zeros_like(v_want))):
        pool = ctx.dev[name].cpu()
        got = pool[pages, :, slots]
        if fmt == "bf16":
            assert ((got.double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol) * (name == "k")).all()
        else:
            scale = ctx.dev[name + "_scale"].cpu()[pages, :, slots]
            if name == "v":
                c, s = P.quantise(flat(want))
                assert np.array_equal(flat(got.view(torch.uint8)), c) and np.array_equal(flat(scale), s)
            else:
                _same_blocks(flat(got.view(torch.uint8)), flat(scale), flat(want), flat(tol), 32)
        touched = torch.zeros(pool.shape[0], pool.shape[2], dtype=torch.bool)
        touched[pages, slots] = True
        assert same(pool.transpose(1, 2)[~touched], before[name].cpu().transpose(1, 2)[~touched])
        if fmt == "e4m3":
            s = name + "_scale"
            assert same(ctx.dev[s].cpu().transpose(1, 2)[~touched], before[s].cpu().transpose(1, 2)[~touched])


# ----------------------------------------------------------------------------- log probabilities
def _place(z, stride, offset):
    """Rows `stride` apart that begin at any element, with NaN around them."""
    n, V = z.shape
    flat = torch.full((n * stride + offset + 64,), float("nan"), dtype=z.dtype, device="cuda")
    rows = flat[offset:offset + n * stride].view(n, stride)[:, :V]
    rows.copy_(z)
    return rows


def _score(E, z, tokens, k, space):
    n = z.shape[0]
    f = lambda *s: torch.full(s, -7.0, device="cuda")                    # noqa: E731
    i = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")   # noqa: E731
    outs = dict(logprob=f(n), entropy=f(n), rank=i(n), top=i(n, k), top_logprob=f(n, k))
    st = _status()
    E.ead_token_logprobs(z, tokens.int(), **outs, workspace=space, status=st)
    return list(outs.values()), st.item()


def _scores(z, tokens, k):
    """The definition in 64 bits, on the device, some rows at a time."""
    out = [[] for _ in range(5)]
    index = torch.arange(z.shape[1], device="cuda")
    for zz, t in zip(z.split(64), tokens.long().split(64)):
        zz, t = zz.double(), t[:, None]
        d = zz - zz.amax(1, keepdim=True)
        logp = d - d.exp().sum(1, keepdim=True).log()
        given = zz.gather(1, t.clamp_min(0))
        rank = ((zz > given) | ((zz == given) & (index < t))).sum(1)
        order = torch.sort(zz + 0.0, dim=1, descending=True, stable=True).indices[:, :k]
        none = t[:, 0] < 0
        out[0].append(torch.where(none, torch.nan, logp.gather(1, t.clamp_min(0))[:, 0]))
        out[1].append(-torch.where(logp.isinf(), 0.0, logp * logp.exp()).sum(1))
        out[2].append(torch.where(none, -1, rank))
        out[3].append(order)
        out[4].append(logp.gather(1, order))
    return [torch.cat(o) for o in out]


def _sum_error(dtype, V, parts=1):
    """Relative error of a row's sum of exponentials.  A thread (256 of a part) adds every other one of its exponentials in turn, half a unit each; an
    exponential is 2^-22 off, and one more for every run of four vectors that brings a new largest logit; 64 roundings for distances
    (2^-24 of up to 40 that matter) and the tree."""
    per_run = 4 * (4 if dtype is torch.float32 else 8)
    per_thread = V / parts / 256
    return (per_thread / 2 + 64) * 2.0 ** -24 + (per_thread / per_run + 3) * 2.0 ** -22


def _check(got, want, z, parts=1):
    """Whole numbers are equal.  Logarithms: the sum's relative error, and three roundings of the numbers that are added.  Entropy ln s - t / s: t has the
    sum's relative error too, and |t / s| is at most ln V."""
    V, err = z.shape[1], _sum_error(z.dtype, z.shape[1], parts)
    top = z.double().masked_fill(z.isinf(), 0.0).abs().amax(1)
    for g, w, tol in ((got[0], want[0], err + 3 * 2.0 ** -24 * (top + math.log(V))), (got[4], want[4], (err + 3 * 2.0 ** -24 * (top + math.log(V)))[:, None]),
                      (got[1], want[1], torch.full_like(top, (err + 2.0 ** -22) * (1 + 2 * math.log(V))))):
        g = g.double()
        same = (g == w) | (g.isnan() & w.isnan())
        tol = tol + 2.0 ** -23 * w.masked_fill(~w.isfinite(), 0.0).abs()
        assert (same | ((g - w).abs() <= tol)).all(), ((g - w).abs() / tol).nan_to_num().max()
    assert torch.equal(got[2].long(), want[2]) and torch.equal(got[3].long(), want[3])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,V,k,offset,stride", [(180, 152064, 64, 0, 152064), (180, 152061, 1, 3, 152067), (300, 40009, 20, 1, 40011), (300, 16385, 0, 5, 16390),
                                                 (300, 24583, 5, 7, 24583)])
def test_token_logprobs_whole_rows(E, space, dtype, n, V, k, offset, stride):
    """More rows than would be cut: a block has all of a row, 2 to 37 runs through its ring, from any alignment."""
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (3.0 * torch.randn(n, V, generator=g, device="cuda")).to(dtype)
    tokens = torch.randint(0, V, (n,), generator=g, device="cuda")
    tokens[:8] = torch.tensor([0, V - 1, -1, V // 2, 9, V - 9, V - 8200, 8200], device="cuda")
    tokens[8:40] = z[8:40].float().argmax(1)
    tokens[40:60] = z[40:60].float().argmin(1)
    z = _place(z, stride, offset)
    got, st = _score(E, z, tokens, k, space)
    assert st == 0
    _check(got, _scores(z, tokens, k), z)


def _contents(V, dtype):
    """Rows that are hard to order or to add up, and whether a row has an answer."""
    g = torch.Generator().manual_seed(V)
    low, tiny, inf = torch.finfo(dtype).min, torch.finfo(dtype).tiny, float("inf")
    r = lambda: torch.randn(V, generator=g)                              # noqa: E731
    z = [torch.zeros(V), torch.randint(0, 3, (V,), generator=g).float(), torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0)]
    z += [r().masked_fill(torch.rand(V, generator=g) < 0.9, -inf), torch.full((V,), -inf), torch.arange(V) * 0.01, torch.arange(V) * -0.01, r()]
    z[4][V // 2] = 2.0
    z[7][V - 1] = 200.0
    z += [torch.full((V,), low), torch.full((V,), low)]
    z[9][::2] = 1.5
    steps = torch.randint(-3, 4, (V,), generator=g).double() * tiny / 4   # numbers below the normal ones, and zeros of both signs
    z += [steps.to(dtype).float(), 1e4 + 50 * r(), r().masked_fill(torch.arange(V) >= 7, -inf)]
    if dtype is not torch.float16:
        z += [2e6 + 1e4 * r(), -7e5 + 1e3 * r(), -3e6 + 1e4 * r(), 1e38 * r(), torch.full((V,), -torch.finfo(dtype).max), 1e37 * r()]
    for at, value in ((V // 3, float("nan")), (V - 5, float("nan")), (9000, inf), (V - 2, inf)):
        z.append(r())
        z[-1][at] = value
    z.append(torch.full((V,), -inf))
    z = torch.stack(z).to(dtype)                                         # (1e38 times a normal number passes the largest one in places)
    return z, ~(z.isnan() | (z == inf)).any(1) & (z > -inf).any(1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,offset", [(40009, 1), (70001, 0)])
def test_token_logprobs_contents_of_whole_rows(E, space, dtype, V, offset):
    """Ties, masks, signed zeros, the ends of the type's range, NaN and infinities in rows that go through the ring."""
    z, ok = _contents(V, dtype)
    kinds = len(z)
    times = -(-160 // kinds)
    z, ok = _place(z.cuda().repeat(times, 1), V + 2, offset), ok.repeat(times).cuda()
    at = torch.tensor([0, V - 1, V // 2, 11, V - 20, V // 3 + 1, 9001, 20000], device="cuda")
    tokens = at[(torch.arange(len(z), device="cuda") // kinds) % len(at)]
    finite = torch.where(ok[:, None], z, torch.zeros((), dtype=dtype, device="cuda"))
    for k in (0, 1, 20, 64):
        want = _scores(finite, tokens, k)
        got, st = _score(E, z, tokens, k, space)
        assert st == E.EAD_STATUS_NONFINITE
        for o in (got[0], got[1], got[4]):
            assert o[~ok].isnan().all()
        assert (got[2][~ok] == -1).all() and (got[3][~ok] == -1).all()
        _check([o[ok] for o in got], [o[ok] for o in want], z[ok])


@pytest.mark.parametrize("dtype", DTYPES)
def test_token_logprobs_counts_every_logit_once(E, space, dtype):
    """Logits of 0: the sum is V exactly, whatever the order; then one logit is missing, at places along the row."""
    n, V = 200, 50000 + 11
    z = _place(torch.zeros(n, V, dtype=dtype, device="cuda"), V + 1, 3)
    at = torch.linspace(0, V - 1, n, device="cuda").long()
    z[torch.arange(1, n, device="cuda"), at[1:]] = -float("inf")
    got, st = _score(E, z, torch.full((n,), V - 1, device="cuda"), 3, space)
    assert st == 0
    count = torch.full((n,), V - 1.0, dtype=torch.float64, device="cuda")
    count[0] = V
    exact = -count.log()
    rest = torch.arange(n, device="cuda") != n - 1                       # (the last row's given token is the one that is masked)
    # the logarithm of an exact number: a unit of 2^-20 in base 2, the constant and the product round to 2^-21 of a number near 11.  1 / V is 2^-15.6
    assert ((got[0].double() - exact).abs()[rest] <= 2.0 ** -18).all() and got[0][n - 1] == -float("inf")
    assert ((got[1].double() + exact).abs() <= 2.0 ** -18).all()
    assert torch.equal(got[2].long(), torch.where(rest & (at != V - 1), V - 2, V - 1).index_fill(0, torch.tensor([0], device="cuda"), V - 1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_token_logprobs_more_rows_than_a_grid(E, space, dtype):
    n, V, k = 65535 + 70, 8201 if dtype is torch.bfloat16 else 4133, 3
    g = torch.Generator(device="cuda").manual_seed(0)
    z = torch.empty(n, V, dtype=dtype, device="cuda")
    for part in z.split(8192):
        part.copy_(2.0 * torch.randn(part.shape, generator=g, device="cuda"))
    tokens = torch.randint(0, V, (n,), generator=g, device="cuda")
    got, st = _score(E, z, tokens, k, space)
    assert st == 0
    for a, b in ((0, 200), (32000, 32200), (65400, n)):
        _check([o[a:b] for o in got], _scores(z[a:b], tokens[a:b], k), z[a:b])
    for a in range(0, n, 8192):                                          # every row's count
        zz, t = z[a:a + 8192].float(), tokens[a:a + 8192, None]
        given = zz.gather(1, t)
        rank = ((zz > given) | ((zz == given) & (torch.arange(V, device="cuda") < t))).sum(1)
        assert torch.equal(rank, got[2][a:a + 8192].long())


@pytest.mark.parametrize("which", ["first", "middle", "last"])
def test_token_logprobs_counts_settle_more_than_once(E, space, which):
    """A row so long that a thread has more than 1024 runs (64 alternatives allow 32 parts: 8.4 million logits each): counts of 16-bit logits are
    settled on the way.  The lowest logit, the largest one and one between are given."""
    V, k = 32 * 1024 * 1024 * 8 + 30_000_011, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.empty(1, V, dtype=torch.bfloat16, device="cuda")
    for part in z[0].split(1 << 25):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    token = dict(first=int(z[0].argmax()), last=V - 3, middle=V // 2 + 5)[which]
    if which == "last":
        z[0, token] = -100.0
    given = z[0, token].item()
    before, total, size = 0, 0.0, 0.0
    top = z.max().item()
    for a in range(0, V, 1 << 25):
        part = z[0, a:a + (1 << 25)]
        before += int((part > given).sum()) + int((part[:max(0, min(len(part), token - a))] == given).sum())
        e = (part.double() - top).exp()
        total += float(e.sum())
    got, st = _score(E, z, torch.tensor([token], device="cuda"), k, space)
    assert st == 0 and got[2].item() == before
    assert abs(got[0].item() - (given - top - math.log(total))) <= _sum_error(torch.bfloat16, V, 32) + 2.0 ** -21 * (1 + abs(given - top) + math.log(total))
    best = torch.sort(z[0], descending=True, stable=True).indices[:k]
    assert torch.equal(got[3][0].long(), best)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,V", [(64, 30001), (200, 30001), (64, 500)])
def test_token_logprobs_says_the_same_twice(E, space, dtype, n, V):
    """A given token that is among the alternatives has one log probability: the two outputs hold the same number."""
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (3.0 * torch.randn(1, V, generator=g, device="cuda")).to(dtype).repeat(n, 1)
    top = _score(E, z, torch.zeros(n, device="cuda"), 64, space)[0][3]
    tokens = top[0].repeat(4)[:n]
    got, _ = _score(E, z, tokens, 64, space)
    assert torch.equal(got[2].long(), torch.arange(64, device="cuda").repeat(4)[:n])
    # (of one row: rows begin at different places in 16 bytes and may be added up in another order)
    assert torch.equal(got[0], got[4].gather(1, got[2].long()[:, None])[:, 0])
