"""The operators of a decoder's 8-bit pass through the Python binding, against plain 64-bit statements of them."""
import numpy as np
import pytest
import torch

import pass_util as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    from paper_2502_06833_b200 import binding
    return binding


@pytest.fixture(scope="module")
def score_space(E):
    return torch.zeros(E.EAD_LOGPROB_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ----------------------------------------------------------------------------- product
def _padded(x, pad):
    """The same values as rows of a wider buffer (which is NaN beside them)."""
    wide = torch.full((x.shape[0], x.shape[1] + pad), 0x7F, dtype=x.dtype)
    wide[:, :x.shape[1]] = x
    return wide.cuda()[:, :x.shape[1]]


class Product:
    """Operands of one product, on the GPU and as 64-bit values."""

    def __init__(self, E, T, N, K, block, seed=0, pad=0, x_size=1.0, edit=None):
        rng = np.random.default_rng(seed)
        spread = lambda n: np.exp2(rng.integers(-6, 7, n))               # noqa: E731  (scales that differ from block to block)
        x = rng.normal(0, x_size, (T, K)) * np.repeat(spread(T * P.up(K, 32)).reshape(T, -1), 32, 1)[:, :K]
        w = rng.normal(0, 1, (N, K)) * np.repeat(np.repeat(spread(P.up(N, 128) * P.up(K, 128)).reshape(-1, P.up(K, 128)), 128, 0)[:N], 128, 1)[:, :K]
        self.x, self.w = [*P.quantise(x, block)], [*P.quantise(w, 128, 128)]
        if edit:
            edit(self)
        self.xv, self.wv = P.values(*self.x, block), P.values(*self.w, 128, 128)
        dev = [torch.from_numpy(a) for a in (*self.x, *self.w)]
        self.mx = E.ead_e4m3_matrix(_padded(dev[0], pad), dev[1].cuda(), block=(1, block))
        self.mw = E.ead_e4m3_matrix(_padded(dev[2], pad), dev[3].cuda(), block=(128, 128))
        self.bias = torch.from_numpy(rng.normal(0, 4, N)).bfloat16().cuda()

    def run(self, E, dtype, bias=True, pad=0, **kw):
        T, N = len(self.xv), len(self.wv)
        out = torch.full((T, -(-N // 8) * 8 + pad), -7.0, dtype=dtype, device="cuda")
        st = _status()
        E.ead_linear(self.mx, self.mw, out[:, :N], bias=self.bias if bias else None, status=st, **kw)
        assert (out[:, N:] == -7.0).all() and st.item() == 0
        return out[:, :N].cpu()

    def check(self, got, bias=True):
        """An instruction adds 32 products to the 32-bit sum, and whatever it drops is below 2^-23 of the magnitudes so far: K / 32 times that,
        the sums of a few parts and the bias; then the rounding of the output, half a step."""
        want = self.xv @ self.wv.T
        size = np.abs(self.xv) @ np.abs(self.wv).T
        if bias:
            b = self.bias.double().cpu().numpy()
            want, size = want + b, size + np.abs(b)
        half = torch.finfo(got.dtype).eps / 2
        tol = (self.xv.shape[1] / 32 + 16) * 2.0 ** -23 * size
        tol = tol + half * (np.abs(want) + tol) + 1e-37
        d = np.abs(got.double().numpy() - want)
        assert not np.isnan(d).any() and (d <= tol).all(), (d / tol).max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("block", [32, 128])
@pytest.mark.parametrize("T,N,K", [(1, 128, 128), (1, 40, 32), (2, 129, 96), (15, 256, 1536), (16, 300, 160), (17, 1000, 512), (64, 7168, 640),
                                   (129, 257, 4128), (240, 384, 256), (241, 130, 1024), (500, 5000, 288), (1000, 1030, 2048)])
def test_linear(E, dtype, block, T, N, K):
    p = Product(E, T, N, K, block, seed=T + N + K)
    p.check(p.run(E, dtype))


@pytest.mark.parametrize("block", [32, 128])
def test_linear_rows_of_wider_buffers(E, block):
    p = Product(E, 37, 203, 416, block, pad=48)
    for bias in (False, True):
        p.check(p.run(E, torch.bfloat16, bias, pad=24), bias)
        p.check(p.run(E, torch.float32, bias, pad=16), bias)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,N,K", [(1, 203, 416), (40, 129, 2048), (241, 301, 128)])
def test_linear_output_rows_anywhere(E, dtype, T, N, K):
    """Rows that begin at any element; what lies before, between and behind them stays."""
    p = Product(E, T, N, K, 128)
    for offset, stride in ((0, N), (1, N + 2), (3, N + 5)):
        flat = torch.full((offset + T * stride + 7,), -7.0, dtype=dtype, device="cuda")
        out = flat[offset:offset + T * stride].view(T, stride)[:, :N]
        E.ead_linear(p.mx, p.mw, out, bias=p.bias)
        p.check(out.cpu())
        out.fill_(-7.0)
        assert (flat == -7.0).all()


@pytest.mark.parametrize("T,N,K", [(1, 2048, 1536), (3, 128, 8192), (64, 1280, 5120), (300, 1300, 4096)])
def test_linear_is_the_same_every_time(E, T, N, K):
    """Tiles cut along K are joined in the order of K, whichever block is slow."""
    p = Product(E, T, N, K, 128)
    first = p.run(E, torch.float32)
    p.check(first)
    for _ in range(20):
        assert torch.equal(p.run(E, torch.float32), first)


@pytest.mark.parametrize("block", [32, 128])
def test_linear_every_scale_reaches_its_block(E, block):
    """Codes of 1 and scales that name their place: the sums are exact in 32 bits."""
    T, N, K = 140, 260, 1152

    def edit(p):
        p.x[0][:], p.w[0][:] = 0x38, 0x38                               # 1.0
        rng = np.random.default_rng(5)
        p.x[1][:] = 127 + rng.integers(-3, 4, p.x[1].shape)
        p.w[1][:] = 127 + rng.integers(-3, 4, p.w[1].shape)
    p = Product(E, T, N, K, block, edit=edit)
    got = p.run(E, torch.float32, bias=False)
    assert np.array_equal(got.double().numpy(), p.xv @ p.wv.T)


def test_linear_far_scales(E):
    """The ends of the scales' range: products that vanish, that stay, and that overflow to infinity."""
    def edit(p):
        p.x[0][:], p.w[0][:] = 0x38, 0x38
        p.x[1][:] = np.array([[7], [127], [246], [246]])
        p.w[1][:] = np.array([[7], [246]])
    p = Product(E, 4, 256, 128, 128, edit=edit)
    got = p.run(E, torch.float32, bias=False).double().numpy()
    want = p.xv @ p.wv.T                                                 # 128 * 2^(a + b)
    want = np.where(want > 3.4e38, np.inf, np.where(want < 2.0 ** -126, 0.0, want))
    assert np.array_equal(np.where(got < 2.0 ** -126, 0.0, got), want)   # below the smallest normal number either 0 or the number


@pytest.mark.parametrize("block", [32, 128])
def test_linear_nan_stays_in_its_row_and_column(E, block):
    def edit(p):
        p.x[0][3, 200] = 0x7F
        p.x[1][70, 1] = 255
        p.x[0][70, block:2 * block] = 0x7F
        p.w[0][130, 5] = 0xFF
        p.w[1][0, 2] = 255
    p = Product(E, 90, 300, 384, block, edit=edit)
    got = p.run(E, torch.bfloat16)
    want = torch.from_numpy(p.xv @ p.wv.T).isnan()
    assert want[3].all() and want[70].all() and want[:, 130].all() and want[:, :128].all() and not want[0, 128:130].any()
    assert torch.equal(got.isnan(), want)


def test_linear_captured_and_replayed(E):
    a, b = Product(E, 9, 700, 1536, 128, seed=1), Product(E, 9, 700, 1536, 128, seed=2)
    out = torch.zeros(9, 704, device="cuda")[:, :700]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        E.ead_linear(a.mx, a.mw, out, stream=side.cuda_stream)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        E.ead_linear(a.mx, a.mw, out, stream=side.cuda_stream)
    g.replay()
    torch.cuda.synchronize()
    a.check(out.cpu(), bias=False)
    for m, o in ((a.mx, b.mx), (a.mw, b.mw)):                            # other operands in the same buffers
        for t, s in zip(m.held, o.held):
            t.copy_(s)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    b.check(out.cpu(), bias=False)


def test_linear_offsets_beyond_32_bits(E):
    """More than 2^31 outputs: the last rows are checked, and that nothing is written behind them."""
    T, N, K = 16500, 131072, 32
    codes, scale = torch.full((T, K), 0x38, dtype=torch.uint8, device="cuda"), torch.full((T, 1), 127, dtype=torch.uint8, device="cuda")
    scale[-1] = 130
    w, ws = torch.full((N, K), 0x38, dtype=torch.uint8, device="cuda"), torch.full((N // 128, 1), 127, dtype=torch.uint8, device="cuda")
    ws[-1] = 128
    out = torch.full((T + 1, N), -1.0, dtype=torch.bfloat16, device="cuda")
    E.ead_linear(E.ead_e4m3_matrix(codes, scale, block=(1, 32)), E.ead_e4m3_matrix(w, ws, block=(128, 128)), out[:T])
    assert (out[T] == -1).all() and (out[0, :-128] == 32).all() and (out[T - 2, :-128] == 32).all()
    assert (out[T - 1, :-128] == 256).all() and (out[T - 1, -128:] == 512).all() and (out[T - 2, -128:] == 64).all()


@pytest.mark.parametrize("T,N,K,block", [(300, 1300, 4096, 128), (500, 1300, 4096, 32), (40, 512, 8192, 32), (5, 5000, 2048, 128), (64, 40000, 512, 128)])
def test_linear_waits_that_run_out(E, T, N, K, block):
    """With a limit of no time waits run out in the middle of sound calls: the kernel ends in order and says so, and the next
    call is right."""
    p = Product(E, T, N, K, block)
    out, st = torch.zeros(T, -(-N // 8) * 8, device="cuda"), _status()
    try:
        for ns in (0, 300, 1000, 3000, 10000):
            E.ead_kv_wait_limit(ns)
            E.ead_linear(p.mx, p.mw, out[:, :N], status=st)
            torch.cuda.synchronize()
        assert st.item() == E.EAD_STATUS_WAIT_EXPIRED
    finally:
        E.ead_kv_wait_limit(-1)
    p.check(p.run(E, torch.float32))


# ----------------------------------------------------------------------------- quantisation
def _same_blocks(codes, scale, y, tol, block, block_rows=1):
    """Codes and scales of values known to within `tol`: what they stand for is no further from y than half a step of the code's spacing (the
    scale's smallest step at least), and the scale is the definition's for some value within tol."""
    lo, hi = P.quantise(np.maximum(np.abs(y) - tol, 0), block, block_rows)[1], P.quantise(np.abs(y) + tol, block, block_rows)[1]
    assert ((scale >= lo) & (scale <= hi)).all()
    v = P.values(codes, scale, block, block_rows)
    y = np.clip(y, -448 * 2.0 ** 119, 448 * 2.0 ** 119)                   # the format's largest value: beyond it they saturate, by definition
    step = np.exp2(scale.astype(np.float64) - 127)
    step = np.repeat(np.repeat(step, block_rows, 0)[:len(y)], block, 1)[:, :y.shape[1]]
    room = np.maximum(2.0 ** -4 * np.abs(y) * (1 + 2.0 ** -4), 2.0 ** -10 * step) + tol
    assert (np.abs(v - y) <= room).all()


@pytest.mark.parametrize("block", [32, 128])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 96), (1, 128), (65, 160), (7, 512), (33, 544), (130, 2016), (5, 13824)])
def test_quantise_rows(E, block, rows, cols):
    """Without a gate the codes are exactly the definition's."""
    rng = np.random.default_rng(rows + cols)
    x = torch.from_numpy(rng.normal(0, 1, (rows, cols)) * np.exp2(rng.integers(-30, 30, (rows, 1)))).bfloat16()
    x[0, :3] = torch.tensor([0.0, -0.0, 1e-38])
    wide = torch.full((rows, cols + 16), float("nan"), dtype=torch.bfloat16)
    wide[:, :cols] = x
    codes = torch.full((rows, cols + 32), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(rows, P.up(cols, block), dtype=torch.uint8, device="cuda")
    E.ead_quantise(wide.cuda()[:, :cols], E.ead_e4m3_matrix(codes[:, :cols], scale, block=(1, block)))
    want = P.quantise(x.double().numpy(), block)
    assert (codes[:, cols:] == 0x55).all()
    assert np.array_equal(codes[:, :cols].cpu().numpy(), want[0]) and np.array_equal(scale.cpu().numpy(), want[1])


@pytest.mark.parametrize("block", [32, 128])
@pytest.mark.parametrize("rows,cols", [(1, 32), (4, 416), (64, 1536), (9, 8960)])
def test_quantise_gated(E, block, rows, cols):
    """silu by the special function unit: the exponential, the sum, the quotient and the product each a few units of 2^-24 off (the
    exponential's error grows with its argument, up to 2^-21 at 88): 2^-19 of the value covers them."""
    rng = np.random.default_rng(cols)
    both = torch.from_numpy(rng.normal(0, 3, (rows, 2, cols))).bfloat16()
    both[0, 0, :8] = torch.tensor([0.0, -0.0, 80.0, -80.0, 300.0, -300.0, 3e38, -3e38])
    codes = torch.zeros(rows, cols, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(rows, P.up(cols, block), dtype=torch.uint8, device="cuda")
    dev = both.cuda()
    E.ead_quantise(dev[:, 1], E.ead_e4m3_matrix(codes, scale, block=(1, block)), gate=dev[:, 0])
    g = both[:, 0].double().numpy()
    with np.errstate(over="ignore"):
        y = both[:, 1].double().numpy() * g / (1 + np.exp(-g))
    _same_blocks(codes.cpu().numpy(), scale.cpu().numpy(), y, 2.0 ** -19 * np.abs(y) + 2.0 ** -125, block)


@pytest.mark.parametrize("rows,cols", [(1, 32), (128, 128), (129, 160), (300, 1056), (77, 4096)])
def test_quantise_tiles(E, rows, cols):
    rng = np.random.default_rng(rows)
    x = torch.from_numpy(rng.normal(0, 1, (rows, cols)) * np.exp2(rng.integers(-9, 9, (1, cols)))).bfloat16()
    codes = torch.zeros(rows, cols, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(P.up(rows, 128), P.up(cols, 128), dtype=torch.uint8, device="cuda")
    E.ead_quantise(x.cuda(), E.ead_e4m3_matrix(codes, scale, block=(128, 128)))
    want = P.quantise(x.double().numpy(), 128, 128)
    assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(scale.cpu().numpy(), want[1])


@pytest.mark.parametrize("block", [(1, 32), (1, 128), (128, 128)])
def test_quantise_not_finite_and_extreme(E, block):
    x = torch.ones(130, 288, dtype=torch.bfloat16)
    x[0, 5], x[1, 40], x[2, 200] = float("nan"), float("inf"), -float("inf")
    x[3] = 0
    x[4], x[5], x[6, :32] = 3.38e38, 1e-40, torch.tensor([448.0, 449.0] * 16)
    x[128, 0], x[129, 287] = 3.38e38, 1e-38
    codes = torch.zeros(130, 288, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(P.up(130, block[0]), P.up(288, block[1]), dtype=torch.uint8, device="cuda")
    E.ead_quantise(x.cuda(), E.ead_e4m3_matrix(codes, scale, block=block))
    want = P.quantise(x.double().numpy(), block[1], block[0])
    assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(scale.cpu().numpy(), want[1])


# ----------------------------------------------------------------------------- norm and rotation
def _inv_freq(rot, base=500000.0):
    return (base ** -(torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float() if rot else torch.zeros(0)


def _rope(E, dim, rot, interleaved, norm, seed):
    g = torch.Generator().manual_seed(seed)
    w = [(1 + 0.3 * torch.randn(dim, generator=g)).bfloat16() if on else None for on in norm]
    f = _inv_freq(rot)
    dev = [None if t is None else t.cuda() for t in w]
    return E.ead_rope(f.cuda(), dim, interleaved=interleaved, q_weight=dev[0], k_weight=dev[1], eps=1e-5), f, w


def _check_rotated(got, want, size):
    """32-bit arithmetic: 16 roundings of the norm and the two products (2^-24 each), the angle to 2^-23 of a half turn and the functions'
    own 2^-22: 2^-19 of the magnitudes; then half a step of bf16."""
    d = (got.double() - want).abs()
    tol = 2.0 ** -19 * size + 2.0 ** -8 * (want.abs() + 2.0 ** -19 * size) + 1e-38
    assert (d <= tol).all(), (d / tol).max()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot,norm", [(128, 128, (1, 1)), (128, 64, (1, 0)), (128, 16, (0, 1)), (64, 64, (0, 0)), (64, 32, (1, 1)), (64, 0, (1, 1)),
                                          (128, 0, (0, 0)), (128, 48, (1, 1))])
@pytest.mark.parametrize("n,hq,hk", [(1, 40, 8), (5, 5, 1), (33, 28, 4), (2, 3, 0), (3, 0, 2), (4, 129, 3)])
def test_qk_norm_rope(E, interleaved, dim, rot, norm, n, hq, hk):
    g = torch.Generator().manual_seed(n * 7 + hq)
    rope, f, w = _rope(E, dim, rot, interleaved, norm, hq)
    place = torch.randint(0, 4000, (n,), generator=g).int()
    place[0] = 2 ** 31 - 1 if n % 2 else -12345
    both = (torch.randn(n, hq + hk + 1, dim, generator=g) * torch.exp(torch.randn(dim, generator=g))).bfloat16()
    dev = both.cuda()                                                    # slices of one wider projection
    q, k = (dev[:, :hq] if hq else None), (dev[:, hq:hq + hk] if hk else None)
    outs = [torch.full((n, h + 1, dim), -7.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hk)]
    E.ead_qk_norm_rope(rope, place.cuda(), q, k, outs[0][:, :hq], outs[1][:, :hk])
    for out, x, weight, h in ((outs[0], both[:, :hq], w[0], hq), (outs[1], both[:, hq:hq + hk], w[1], hk)):
        assert (out[:, h:] == -7.0).all()
        if h:
            _check_rotated(out[:, :h].cpu(), *P.rotated(x, weight, place, f, interleaved, 1e-5))
    if hq and hk:                                                        # in place
        E.ead_qk_norm_rope(rope, place.cuda(), q, k, q, k)
        assert torch.equal(q, outs[0][:, :hq]) and torch.equal(k, outs[1][:, :hk]) and torch.equal(dev[:, hq + hk:].cpu(), both[:, hq + hk:])


def test_rope_rows_of_zeros_and_not_finite(E):
    rope, f, w = _rope(E, 64, 64, False, (1, 1), 0)
    x = torch.randn(4, 3, 64, generator=torch.Generator().manual_seed(0)).bfloat16()
    x[0, 1] = 0
    x[1, 2, 7], x[2, 0, 60] = float("nan"), float("inf")
    out = torch.zeros(4, 3, 64, dtype=torch.bfloat16, device="cuda")
    E.ead_qk_norm_rope(rope, torch.arange(4, dtype=torch.int32, device="cuda"), x.cuda(), None, out, None)
    assert (out[0, 1] == 0).all() and out[1, 2].isnan().all()
    bad = torch.zeros(4, 3, dtype=torch.bool)
    bad[1, 2] = bad[2, 0] = True
    assert not out.cpu()[~bad].isnan().any()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["head", "token", "padded"])
@pytest.mark.parametrize("hq,heads,dim,page,interleaved,rot", [(8, 2, 128, 16, False, 128), (5, 1, 64, 8, True, 64), (9, 3, 64, 32, False, 32),
                                                               (56, 8, 128, 64, False, 128)])
@pytest.mark.parametrize("far", [False, True])
def test_kv_rotate_write(E, fmt, layout, hq, heads, dim, page, interleaved, rot, far):
    """Queries, keys and values of a ragged step; what the cache held elsewhere stays as it was."""
    from decoder_util import Context
    new, length = [1, 0, 37, 5, 1], [1, 9, 50, 300, 16]
    ctx = Context(new, length, heads, dim, page, fmt, seed=hq, layout=layout, stale=0.25)
    n = sum(new)
    g = torch.Generator().manual_seed(hq)
    both = (torch.randn(n, hq + 2 * heads, dim, generator=g) * torch.exp(0.5 * torch.randn(dim, generator=g))).bfloat16()
    dev = both.cuda()
    rope, f, w = _rope(E, dim, rot, interleaved, (1, 1), 3)
    place = torch.cat([torch.arange(l - m, l) for m, l in zip(new, length)]).int()
    at = place if not far else place + 1000000
    before = {s: t.clone() for s, t in ctx.dev.items()}
    out, st = torch.zeros(n, hq, dim, dtype=torch.bfloat16, device="cuda"), _status()
    E.ead_kv_rotate_write(rope, ctx.cache(E), ctx.batch(E), dev[:, :hq], dev[:, hq:hq + heads], dev[:, hq + heads:], out,
                          positions=at.cuda() if far else None, status=st)
    assert st.item() == 0
    _check_rotated(out.cpu(), *P.rotated(both[:, :hq], w[0], at, f, interleaved, 1e-5))
    owner = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new))
    pages, slots = torch.from_numpy(ctx.table)[owner, place.long() // page].long(), place.long() % page
    k_want, k_size = P.rotated(both[:, hq:hq + heads], w[1], at, f, interleaved, 1e-5)
    v_want = both[:, hq + heads:].double()
    for name, want, tol in (("k", k_want, 2.0 ** -19 * k_size), ("v", v_want, torch.zeros_like(v_want))):
        pool = ctx.dev[name].cpu()
        got = pool[pages, :, slots]
        if fmt == "bf16":
            d = (got.double() - want).abs()
            assert (d <= tol + 2.0 ** -8 * (want.abs() + tol) * (name == "k")).all()
        else:
            scale = ctx.dev[name + "_scale"].cpu()[pages, :, slots]
            codes = got.view(torch.uint8)
            flat = lambda t: t.reshape(-1, t.shape[-1]).numpy()           # noqa: E731
            if name == "v":
                c, s = P.quantise(flat(want))
                assert np.array_equal(flat(codes), c) and np.array_equal(flat(scale), s)
            else:
                _same_blocks(flat(codes), flat(scale), flat(want), flat(tol), 32)
        touched = torch.zeros(pool.shape[0], pool.shape[2], dtype=torch.bool)
        touched[pages, slots] = True
        old = before[name].cpu()
        same = lambda a, b: torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))   # noqa: E731
        assert same(pool.transpose(1, 2)[~touched], old.transpose(1, 2)[~touched])
        if fmt == "e4m3":
            assert same(ctx.dev[name + "_scale"].cpu().transpose(1, 2)[~touched], before[name + "_scale"].cpu().transpose(1, 2)[~touched])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_kv_rotate_write_tokens_without_a_place(E, fmt):
    """Bad pages, contradicting counts and rows behind the last sequence: nothing of such a token is written, the others are."""
    from decoder_util import Context
    new, length = [4, 3, 2], [20, 3, 40]
    ctx = Context(new, length, 2, 64, 16, fmt, stale=0.25)
    rope, f, w = _rope(E, 64, 64, False, (1, 1), 3)
    x = torch.randn(9, 8, 64, generator=torch.Generator().manual_seed(0)).bfloat16().cuda()

    def go(**kw):
        out, st = torch.full((kw.get("n_tokens", 9), 4, 64), -7.0, dtype=torch.bfloat16, device="cuda"), _status()
        n = len(out)
        E.ead_kv_rotate_write(rope, ctx.cache(E), ctx.batch(E, **kw), x[:n, :4], x[:n, 4:6], x[:n, 6:], out, status=st)
        return (out == -7.0).flatten(1).all(1).cpu(), st.item()
    skipped, st = go()
    assert st == 0 and not skipped.any()
    ctx.d_table[1, 0] = 1 << 29
    skipped, st = go()
    assert st == E.EAD_STATUS_BAD_PAGE and skipped.tolist() == [False] * 4 + [True] * 3 + [False] * 2
    ctx.d_table[1, 0] = int(ctx.table[1, 0])
    before = {s: t.clone() for s, t in ctx.dev.items()}
    ctx.d_new_start.copy_(torch.tensor([0, 4, 4, 6], dtype=torch.int32))   # the last three tokens belong to nobody
    skipped, st = go()
    assert st == E.EAD_STATUS_BAD_COUNT and skipped.tolist() == [False] * 6 + [True] * 3
    ctx.d_new_start.copy_(torch.tensor([0, 7, 7, 9], dtype=torch.int32))   # seven tokens where four are allowed
    for s, t in ctx.dev.items():
        t.copy_(before[s])
    skipped, st = go(max_new=4)
    assert st == E.EAD_STATUS_BAD_COUNT and skipped.tolist() == [True] * 7 + [False] * 2
    ctx.d_len[0] = 2                                                     # positions before the context's begin
    ctx.d_new_start.copy_(torch.tensor([0, 4, 7, 9], dtype=torch.int32))
    skipped, st = go()
    assert st == E.EAD_STATUS_BAD_PAGE and skipped.tolist() == [True] * 2 + [False] * 7


# ----------------------------------------------------------------------------- log probabilities
def _score(E, z, tokens, k, score_space, stride=None, offset=0, **kw):
    n, V = z.shape
    flat = torch.full((n * (stride or V) + offset + 64,), float("nan"), dtype=z.dtype)
    rows = flat[offset:offset + n * (stride or V)].view(n, -1)[:, :V]
    rows.copy_(z)
    dev = flat.cuda()[offset:offset + n * (stride or V)].view(n, -1)[:, :V]
    f = lambda *s: torch.full(s, -7.0, device="cuda")                    # noqa: E731
    i = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")   # noqa: E731
    outs = dict(logprob=f(n), entropy=f(n), rank=i(n), top=i(n, k), top_logprob=f(n, k))
    st = _status()
    E.ead_token_logprobs(dev, tokens.int().cuda(), **outs, workspace=score_space, status=st, **kw)
    return [o.cpu() for o in outs.values()], st.item()


def _check_scores(got, want, z):
    """Whole numbers are equal.  A sum of V exponentials in any tree: 2^-24 each level and 2^-22 for an exponential, on a distance
    that is rounded once (2^-24 of it); log probabilities then add three roundings of their own size.  Entropy: s and t come with the same
    relative errors, t / s is bounded by the entropy plus ln V."""
    V = z.shape[1]
    size = torch.where(z.isinf(), torch.zeros(()).double(), z).abs().amax(1)
    for g, w, scale in ((got[0], want[0], size), (got[1], want[1], torch.full_like(size, np.log(V) + 1)), (got[4], want[4], size[:, None])):
        g = g.double()
        same = (g == w) | (g.isnan() & w.isnan())
        tol = 2.0 ** -20 * (1 + torch.where(w.isfinite(), w, torch.zeros(()).double()).abs() + scale)
        assert (same | ((g - w).abs() <= tol)).all(), ((g - w).abs() / tol).nan_to_num().max()
    assert torch.equal(got[2].long(), want[2]) and torch.equal(got[3].long(), want[3])


def _logits(n, V, dtype, seed=0, size=3.0):
    g = torch.Generator().manual_seed(seed)
    z = size * torch.randn(n, V, generator=g)
    z[:, torch.randint(0, V, (20,), generator=g)] += 6.0
    return z.to(dtype), torch.randint(0, V, (n,), generator=g)


DTYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,V,k", [(1, 128256, 5), (1, 1, 1), (3, 7, 20), (2, 64, 64), (300, 1000, 8), (5, 4097, 0), (1, 50257, 64), (40, 9001, 20),
                                   (7, 151665, 1), (150, 8200, 5), (1, 8193, 3)])
def test_token_logprobs(E, score_space, dtype, n, V, k):
    z, tokens = _logits(n, V, dtype, seed=V + k)
    tokens[0] = z[0].float().argmax()
    if n > 1:
        tokens[1] = -1
    got, st = _score(E, z, tokens, k, score_space)
    assert st == 0
    _check_scores(got, P.scores(z.double(), tokens, k), z.double())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset,stride", [(1, 1003), (3, 1000), (8, 1016), (5, 1001)])
def test_token_logprobs_rows_anywhere(E, score_space, dtype, offset, stride):
    """Rows that begin at any element; what lies between and behind them is NaN."""
    z, tokens = _logits(6, 1000, dtype, seed=offset)
    got, st = _score(E, z, tokens, 8, score_space, stride=stride, offset=offset)
    assert st == 0
    _check_scores(got, P.scores(z.double(), tokens, 8), z.double())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [600, 40000])
def test_token_logprobs_ties_and_masks(E, score_space, dtype, V):
    """Equal logits everywhere (more than any list holds), few values, signed zeros, masks of -infinity and of the type's lowest value, sorted
    rows both ways, one token certain."""
    low = torch.finfo(dtype).min
    g = torch.Generator().manual_seed(V)
    z = torch.zeros(9, V)
    z[1] = torch.randint(0, 3, (V,), generator=g).float()
    z[2] = torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0)
    z[3] = torch.randn(V, generator=g)
    z[3, torch.rand(V, generator=g) < 0.9] = -float("inf")
    z[4] = -float("inf")
    z[4, V // 2] = 2.0
    z[5] = torch.arange(V) * 0.01
    z[6] = -torch.arange(V) * 0.01
    z[7, V - 1] = 200.0
    z = z.to(dtype)
    z[8] = low
    for shift in (0, V // 3, V - 1):
        tokens = torch.full((9,), shift)
        for k in (0, 1, 20, 64):
            got, st = _score(E, z, tokens, k, score_space)
            assert st == 0
            want = P.scores(z.double(), tokens, k)
            _check_scores(got, want, torch.where(z.double() <= low, torch.zeros(()).double(), z.double()))
    z[8, ::2] = 1.5
    got, st = _score(E, z, tokens, 20, score_space)
    _check_scores(got, P.scores(z.double(), tokens, 20), torch.where(z.double() <= low, torch.zeros(()).double(), z.double()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,V", [(5, 1000), (2, 60000)])
def test_token_logprobs_rows_that_say_nothing(E, score_space, dtype, n, V):
    z, tokens = _logits(n, V, dtype)
    bad = torch.zeros(n, dtype=torch.bool)
    z[0, V - 3] = float("nan")
    z[1, 2] = float("inf")
    bad[:2] = True
    if n > 2:
        z[2] = -float("inf")
        z[3, 0] = -float("inf")
        bad[2] = True
    got, st = _score(E, z, tokens, 5, score_space)
    assert st == E.EAD_STATUS_NONFINITE
    assert got[0][bad].isnan().all() and got[1][bad].isnan().all() and got[4][bad].isnan().all()
    assert (got[2][bad] == -1).all() and (got[3][bad] == -1).all()
    if n > 2:
        ok = ~bad
        _check_scores([o[ok] for o in got], P.scores(z[ok].double(), tokens[ok], 5), z[ok].double())
    z, tokens = _logits(n, V, dtype)
    tokens[0], tokens[1] = V, -5
    got, st = _score(E, z, tokens, 5, score_space)
    assert st == E.EAD_STATUS_BAD_TOKEN
    assert got[0][:2].isnan().all() and (got[2][:2] == -1).all() and got[1].isfinite().all() and (got[3] >= 0).all()


def test_token_logprobs_some_outputs_only(E, score_space):
    z, tokens = _logits(3, 5000, torch.bfloat16)
    want = P.scores(z.double(), tokens, 7)
    dev, t = z.cuda(), tokens.int().cuda()
    top = torch.zeros(3, 7, dtype=torch.int32, device="cuda")
    E.ead_token_logprobs(dev, None, top=top, workspace=score_space)
    assert torch.equal(top.cpu().long(), want[3])
    rank = torch.zeros(3, dtype=torch.int32, device="cuda")
    E.ead_token_logprobs(dev, t, rank=rank, workspace=score_space)
    assert torch.equal(rank.cpu().long(), want[2])
    lp = torch.zeros(3, 7, device="cuda")
    E.ead_token_logprobs(dev, None, top_logprob=lp, workspace=score_space)
    assert (lp.cpu().double() - want[4]).abs().max() < 1e-4
    h = torch.zeros(3, device="cuda")
    E.ead_token_logprobs(dev, t, entropy=h, workspace=score_space)
    assert (h.cpu().double() - want[1]).abs().max() < 1e-4


def test_token_logprobs_is_the_same_every_time_and_replays(E, score_space):
    z, tokens = _logits(2, 100000, torch.float32)
    first, _ = _score(E, z, tokens, 20, score_space)
    for _ in range(10):
        again, _ = _score(E, z, tokens, 20, score_space)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    dev, t = z.cuda(), tokens.int().cuda()
    h = torch.zeros(2, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        E.ead_token_logprobs(dev, t, entropy=h, workspace=score_space, stream=side.cuda_stream)
    dev.copy_(dev.flip(0))
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(h.cpu(), first[1].flip(0))
