"""The decoder-side operators through the Python binding, against plain 64-bit statements of them."""
import numpy as np
import pytest
import torch

from decoder_util import Context, attention, quantise, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    from paper_2502_06833_b200 import binding
    return binding


@pytest.fixture(scope="module")
def workspace(E):
    return torch.zeros(E.EAD_KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _attend(E, ctx, q, workspace, scale, window=0, sinks=0, pad=0, **kw):
    """Runs the entry point; with `pad` the rows of q and out lie apart, as slices of a wider buffer."""
    n, hq, dim = q.shape
    wide = torch.full((n, hq + pad, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :hq] = q.cuda()
    out = torch.full((n, hq + pad, dim), -7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, hq), -7.0, device="cuda")
    st = _status()
    E.ead_kv_attention(ctx.cache(E), ctx.batch(E, **kw), wide[:, :hq], out[:, :hq], scale=scale, window=window, sinks=sinks,
                       lse=lse, workspace=workspace, status=st, stream=_stream())
    assert (out[:, hq:] == -7.0).all()
    return out[:, :hq].cpu(), lse.cpu(), st.item()


def _check(got, want):
    out, lse, status = got
    w_out, w_lse, tol_o, tol_l = want
    assert status == 0
    bad = (out.double() - w_out).abs() > tol_o
    assert not bad.any() and not out.isnan().any(), (int(bad.sum()), ((out.double() - w_out).abs() / tol_o).max())
    fin = torch.isfinite(w_lse)
    assert torch.equal(lse[~fin].double(), w_lse[~fin])
    d = (lse.double() - w_lse).abs()
    assert (d[fin] <= tol_l[fin]).all(), (d[fin] / tol_l[fin]).max()


def _q(ctx, group, seed=1, size=1.5):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn(int(ctx.new_start[-1]), ctx.heads * group, ctx.dim, generator=g)).bfloat16()


ONE = [1] * 9
LENS = [1, 2, 15, 16, 17, 31, 129, 300, 1025]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,group,dim,page", [(2, 4, 128, 16), (8, 4, 64, 16), (2, 5, 128, 32), (1, 8, 128, 64), (3, 1, 64, 8),
                                                  (2, 7, 128, 128), (2, 16, 128, 256), (1, 9, 64, 32)])
def test_attention_single_tokens(E, workspace, fmt, heads, group, dim, page):
    ctx = Context(ONE, LENS, heads, dim, page, fmt, seed=heads * 100 + group)
    q = _q(ctx, group)
    _check(_attend(E, ctx, q, workspace, dim ** -0.5), attention(ctx, q, dim ** -0.5, 0, 0))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,group,dim,page", [(2, 4, 128, 16), (2, 4, 64, 32), (1, 5, 128, 64), (2, 1, 128, 128), (1, 7, 64, 8),
                                                  (1, 71, 64, 16), (1, 128, 128, 256)])
@pytest.mark.parametrize("new,length", [([5, 33, 64, 200, 1, 0, 129], [5, 40, 500, 200, 77, 60, 900]),
                                        ([257, 1], [1000, 4000])])
def test_attention_chunks(E, workspace, fmt, heads, group, dim, page, new, length):
    if group > 16:
        new, length = [min(n, 40) for n in new], length
    ctx = Context(new, length, heads, dim, page, fmt, seed=group)
    q = _q(ctx, group)
    _check(_attend(E, ctx, q, workspace, dim ** -0.5), attention(ctx, q, dim ** -0.5, 0, 0))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 1), (100, 4), (128, 128), (200, 0), (129, 300), (5000, 4)])
@pytest.mark.parametrize("new,length,group,dim,page", [([1, 1, 1, 1], [1, 130, 700, 2000], 4, 128, 16),
                                                       ([3, 2, 300, 60], [3, 650, 1000, 200], 5, 128, 32),
                                                       ([128, 40], [1200, 40], 2, 64, 64)])
def test_attention_window_and_sinks(E, workspace, fmt, window, sinks, new, length, group, dim, page):
    ctx = Context(new, length, 2, dim, page, fmt, seed=window)
    q = _q(ctx, group)
    _check(_attend(E, ctx, q, workspace, 0.11, window, sinks), attention(ctx, q, 0.11, window, sinks))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,group", [([1, 1, 1], 4), ([1, 100, 30], 4)])
def test_attention_does_not_touch_what_no_query_sees(E, workspace, fmt, new, group):
    """Keys before every window (and past the sinks) hold NaN, and their pages' table entries are invalid."""
    length, window, sinks, page = [700, 900, 333], 64, 3, 16
    lows = [l - n - window + 1 for n, l in zip(new, length)]

    def fill(name, b, x):
        x[sinks:max(sinks, lows[b])] = float("nan")
        return x
    ctx = Context(new, length, 2, 128, page, fmt, seed=3, fill=fill)
    for b, lo in enumerate(lows):
        ctx.table[b, -(-sinks // page):lo // page] = -5
    ctx.d_table = torch.from_numpy(ctx.table).cuda()
    q = _q(ctx, group)
    got = _attend(E, ctx, q, workspace, 0.1, window, sinks)
    for name in "kv":
        ctx.host[name] = [torch.nan_to_num(x) for x in ctx.host[name]]
    _check(got, attention(ctx, q, 0.1, window, sinks))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attention_rows_that_see_nothing(E, workspace, fmt):
    """Contexts shorter than the chunk: the first queries have negative positions."""
    ctx = Context([1, 4, 40, 200, 3], [0, 1, 13, 150, 3], 2, 128, 16, fmt, seed=4)
    q = _q(ctx, 4)
    got = _attend(E, ctx, q, workspace, 0.1)
    want = attention(ctx, q, 0.1, 0, 0)
    assert torch.isneginf(want[1]).sum() == (1 + 3 + 27 + 50) * 8
    assert (got[0][torch.isneginf(want[1])] == 0).all()
    _check(got, want)


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 30, 7), (3, 2 ** 31 - 1)])
def test_attention_extreme_windows_with_rows_that_see_nothing(E, workspace, window, sinks):
    """The largest windows and sinks next to negative positions and a negative context length."""
    ctx = Context([4, 40, 1, 200], [1, 13, 700, 150], 2, 128, 16, seed=16)
    q = _q(ctx, 4)
    _check(_attend(E, ctx, q, workspace, 0.1, window, sinks), attention(ctx, q, 0.1, min(window, 10 ** 6), min(sinks, 10 ** 6)))
    ctx.d_len[0] = -5                                   # counts as no context
    ctx.length[0] = 0
    out, lse, st = _attend(E, ctx, q, workspace, 0.1, window, sinks, max_len=700)
    assert st == 0 and (out[:4] == 0).all() and torch.isneginf(lse[:4]).all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["token", "padded"])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_strides(E, workspace, fmt, layout, dim):
    ctx = Context([1, 70, 2, 1], [90, 500, 33, 260], 2, dim, 16, fmt, seed=5, layout=layout)
    q = _q(ctx, 4)
    _check(_attend(E, ctx, q, workspace, 0.1, pad=3), attention(ctx, q, 0.1, 0, 0))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 60])
def test_attention_with_meaningless_strides(E, workspace, dim, new):
    """One cache head, one page: the strides of those dimensions may be anything."""
    ctx = Context([new], [200], 1, dim, 256, seed=21)
    q = _q(ctx, 4)
    want = attention(ctx, q, 0.1, 0, 0)
    page = int(ctx.table[0, 0])
    for name in "kv":
        ctx.dev[name] = ctx.dev[name][page:page + 1].as_strided((1, 1, 256, dim), (7 if name == "k" else 8, 3, dim, 1),
                                                                ctx.dev[name][page].storage_offset())
    ctx.table[:] = 0
    ctx.d_table = torch.zeros(1, 1, dtype=torch.int32, device="cuda").as_strided((1, 1), (1, 5))
    _check(_attend(E, ctx, q, workspace, 0.1), want)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attention_long_context_split_over_many_blocks(E, workspace, fmt):
    """One sequence over all the GPU's blocks; repeated calls agree bit for bit and reuse the workspace."""
    ctx = Context([1], [30011], 1, 128, 32, fmt, seed=6)
    q = _q(ctx, 4)
    first = _attend(E, ctx, q, workspace, 0.09)
    _check(first, attention(ctx, q, 0.09, 0, 0))
    for _ in range(5):
        again = _attend(E, ctx, q, workspace, 0.09)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    ctx = Context([100], [9000], 1, 128, 32, fmt, seed=7)
    q = _q(ctx, 4)
    first = _attend(E, ctx, q, workspace, 0.09)
    _check(first, attention(ctx, q, 0.09, 0, 0))
    for _ in range(5):
        again = _attend(E, ctx, q, workspace, 0.09)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,length,heads,group,dim,page,window,sinks", [
    ([1], [30011], 1, 4, 128, 32, 0, 0), ([1], [20011], 1, 8, 64, 16, 0, 0), ([3], [20011], 1, 4, 128, 64, 0, 0),
    ([100], [9000], 1, 4, 128, 32, 0, 0), ([20], [9003], 2, 4, 64, 16, 0, 0), ([150, 1], [6000, 9000], 1, 5, 128, 16, 0, 0),
    ([1, 70], [12000, 9000], 1, 4, 128, 16, 5000, 300), ([40], [5000], 1, 20, 64, 128, 0, 0)])
def test_every_value_tile_counts_once(E, workspace, fmt, new, length, heads, group, dim, page, window, sinks):
    """Work split over many blocks: keys 16 i .. 16 i + 15 have value 1 in dimension i % head_dim and 0 elsewhere, and logits are
    nearly flat, so a run of 16 values that is lost or counted twice moves its dimension by far more than the tolerance.
    That it does is checked on the 64-bit result."""
    def fill(name, b, x):
        if name == "v":
            x = torch.zeros_like(x)
            key = torch.arange(len(x))
            x[key, :, key // 16 % dim] = 1.0
        return x
    ctx = Context(new, length, heads, dim, page, fmt, seed=18, fill=fill)
    q = _q(ctx, group, size=0.3)
    scale = dim ** -0.5
    want = attention(ctx, q, scale, window, sinks)
    t = 0
    for b, (m, l) in enumerate(zip(new, length)):
        pos = l - 1                                            # the sequence's last query, all of whose heads are looked at
        seen = torch.arange(l)
        seen = (seen > pos - window) | (seen < sinks) if window else seen <= pos
        for hq in range(heads * group):
            z = scale * (ctx.host["k"][b][:, hq // group] @ q[t + m - 1, hq].double())
            w = torch.softmax(torch.where(seen, z, torch.full((), -np.inf, dtype=torch.float64)), 0)[:l // 16 * 16].view(-1, 16)
            whole = seen[:l // 16 * 16].view(-1, 16).all(1)
            assert (w.sum(1) > 2 * want[2][t + m - 1, hq][torch.arange(l // 16) % dim])[whole].all()
        t += m
    _check(_attend(E, ctx, q, workspace, scale, window, sinks), want)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("size,trend", [(8.0, 0.0), (3.0, 1.0), (3.0, -1.0), (60.0, 0.0)])
@pytest.mark.parametrize("new", [1, 140])
def test_attention_wide_logits(E, workspace, fmt, size, trend, new):
    """Logits of a wide range, and maxima that rise or fall along the context (every tile moves the maximum)."""
    def fill(name, b, x):
        if name == "k":
            ramp = torch.linspace(-1, 1, x.shape[0])[:, None, None] * trend
            x = (x.float() * 0.3 + 3 * ramp).bfloat16() if trend else x
        return x
    ctx = Context([new, new], [1500, 777], 2, 128, 16, fmt, seed=8, fill=fill)
    q = _q(ctx, 4, size=size)
    if trend:
        q = q.abs()
    _check(_attend(E, ctx, q, workspace, 0.1), attention(ctx, q, 0.1, 0, 0))


def test_attention_e4m3_scales_over_their_whole_range(E, workspace):
    """Blocks whose scales lie anywhere from 2^-120 to far above 1 (keys stay small where values are large)."""
    powers = [-125, -100, -40, -3, 0, 9, 17, 60]

    def fill(name, b, x):
        if name == "v":
            x = x * 2.0 ** powers[b]
        return x.bfloat16()
    for new in (1, 50):
        ctx = Context([new] * 8, [200] * 8, 1, 128, 16, "e4m3", seed=9, fill=fill)
        q = _q(ctx, 4)
        want = attention(ctx, q, 0.1, 0, 0)
        tiny = torch.full((), 2.0 ** -126, dtype=torch.float64)                 # bf16 results below the normal range
        _check(_attend(E, ctx, q, workspace, 0.1), (want[0], want[1], torch.maximum(want[2], tiny), want[3]))

    def fill_k(name, b, x):
        return (x * 2.0 ** (10 if name == "k" else 0)).bfloat16()
    for new in (1, 50):
        ctx = Context([new] * 2, [200] * 2, 1, 128, 16, "e4m3", seed=10, fill=fill_k)
        q = _q(ctx, 4, size=2.0 ** -9)
        _check(_attend(E, ctx, q, workspace, 0.1), attention(ctx, q, 0.1, 0, 0))


@pytest.mark.parametrize("new", [1, 2, 50])
def test_attention_e4m3_small_codes_mixed_scales_and_large_queries(E, workspace, new):
    """Blocks whose values but one are subnormal codes, neighbouring keys with scales 2^40 apart (also above
    2^-2, where the probabilities cannot take them in), and query rows of very different size."""
    def fill(name, b, x):
        y = x.float()
        if b == 0:
            y = y * 2.0 ** -14
            y[:, :, ::32] = 0.4
        elif b == 1 and name == "v":
            y = y * torch.where(torch.arange(len(y)) % 3 == 0, 2.0 ** -30, 2.0 ** 10)[:, None, None]
        elif b == 2 and name == "v":
            y = y * torch.where(torch.arange(len(y)) % 2 == 0, 2.0 ** 90, 1.0)[:, None, None]
        elif b == 3 and name == "k":
            y = y * torch.where(torch.arange(y.shape[2]) < 32, 2.0 ** -20, 2.0 ** -3)
        return y.bfloat16()
    ctx = Context([new] * 5, [333, 200, 77, 500, 140], 2, 128, 16, "e4m3", seed=14, fill=fill)
    q = _q(ctx, 4)
    q[4 * new:, :, 5] *= 2.0 ** 4                      # one element far above the rest of its row
    q[4 * new:, :, 6:] *= 2.0 ** -20
    _check(_attend(E, ctx, q, workspace, 0.02), attention(ctx, q, 0.02, 0, 0))


@pytest.mark.parametrize("new", [1, 50])
def test_attention_nan_blocks_reach_only_their_sequence(E, workspace, new):
    """A value block with an infinity is NaN for its 32 dimensions and its own sequence and head only."""
    def fill(name, b, x):
        if b == 1 and name == "v":
            x[3, 1, 40] = float("inf")
        return x
    for fmt in ("e4m3",):
        ctx = Context([new] * 3, [120, 130, 140], 2, 128, 16, fmt, seed=15, fill=fill)
        q = _q(ctx, 4)
        out, lse, st = _attend(E, ctx, q, workspace, 0.1)
        assert st == 0 and torch.isfinite(lse).all()
        nan = torch.zeros_like(out, dtype=torch.bool)
        nan[new:2 * new, 4:, 32:64] = True
        assert torch.equal(out.isnan(), nan)


def test_attention_on_another_stream_and_in_a_graph(E, workspace):
    ctx = Context([1, 90], [900, 1000], 2, 128, 16, seed=11)
    q = _q(ctx, 4)
    want = attention(ctx, q, 0.1, 0, 0)
    cache, batch = ctx.cache(E), ctx.batch(E)
    dq = q.cuda()
    out, lse, st = torch.empty_like(dq), torch.empty(dq.shape[:2], device="cuda"), _status()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call = lambda s: E.ead_kv_attention(cache, batch, dq, out, scale=0.1, lse=lse, workspace=workspace, status=st, stream=s)  # noqa: E731
    call(side.cuda_stream)
    side.synchronize()
    _check((out.cpu(), lse.cpu(), st.item()), want)
    out.fill_(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    _check((out.cpu(), lse.cpu(), st.item()), want)


@pytest.mark.parametrize("fmt,new,length,heads,dim,runs_out", [
    ("bf16", [1] * 64, [1024 + 113 * b for b in range(64)], 8, 128, False), ("e4m3", [1] * 64, [1024 + 113 * b for b in range(64)], 8, 128, False),
    ("bf16", [300], [30000], 8, 128, True), ("e4m3", [300], [30000], 8, 128, True), ("bf16", [300, 1], [30000, 9000], 8, 64, True),
    ("e4m3", [1, 40, 300, 17], [20000, 5000, 30000, 17], 4, 64, True)])
def test_attention_waits_that_run_out(E, fmt, new, length, heads, dim, runs_out):
    """With limits far below what loads under full load and whole units take, waits run out in the middle of everything: the call
    ends, says so and writes nowhere but into its rows, and with a cleared workspace the next call is sound.  (A single
    look at a barrier lasts several microseconds, about what a copy takes under full load: the few-rows kernel's waits, all of
    them for copies, may or may not run out.)"""
    g = torch.Generator(device="cuda").manual_seed(20)
    page, group = 16, 4
    pages = [-(-n // page) for n in length]
    table = torch.zeros(len(new), max(pages), dtype=torch.int32)
    order, at = torch.randperm(sum(pages), generator=torch.Generator().manual_seed(20)).int(), 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (sum(pages), heads, page, dim)
    if fmt == "bf16":
        pools = [torch.randn(shape, generator=g, device="cuda").bfloat16() for _ in "kv"]
    else:
        pools = [torch.randint(0, 0x7F, shape, generator=g, device="cuda", dtype=torch.uint8) for _ in "kv"]
        pools += [torch.randint(112, 119, (*shape[:3], dim // 32), generator=g, device="cuda", dtype=torch.uint8) for _ in "kv"]
    before = [x.clone() for x in pools]
    n = sum(new)
    starts = torch.tensor([0] + new).cumsum(0).int().cuda()
    batch = E.ead_kv_batch(table.cuda(), starts, torch.tensor(length, dtype=torch.int32, device="cuda"), n_tokens=n, max_new=max(new),
                           max_len=max(length))
    cache = E.ead_kv_cache(*pools)
    q = torch.randn(n, heads * group, dim, generator=g, device="cuda").bfloat16()
    ws = torch.zeros(E.EAD_KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")

    def call(limit):
        out = torch.full((n, heads * group + 1, dim), -7.0, dtype=torch.bfloat16, device="cuda")
        lse, st = torch.full((n, heads * group), -7.0, device="cuda"), _status()
        E.ead_kv_wait_limit(limit)
        try:
            E.ead_kv_attention(cache, batch, q, out[:, :-1], scale=0.1, lse=lse, workspace=ws, status=st, stream=_stream())
        finally:
            E.ead_kv_wait_limit(-1)
        assert (out[:, -1] == -7.0).all()
        if st.item():
            assert st.item() == E.EAD_STATUS_WAIT_EXPIRED
            ws.zero_()
        return out, lse, st.item()
    sound = call(-1)
    assert sound[2] == 0
    seen = set()
    for limit in (20000, 8000, 4000, 2000, 1000, 500, 100, 0, 0, 0, -1):
        got = call(limit)
        seen.add(got[2])
        if got[2] == 0:
            assert torch.equal(got[0], sound[0]) and torch.equal(got[1], sound[1])
    assert got[2] == 0 and (len(seen) == 2 or not runs_out)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(pools, before))


def test_attention_of_more_tiles_than_a_block_counts_is_refused(E, workspace):
    """4096 sequences of up to 2^30 keys with 128 cache heads; nothing is launched, so nothing of it exists."""
    import ctypes as C
    k = torch.zeros(1, 128, 256, 64, dtype=torch.bfloat16, device="cuda")
    cache = E.ead_kv_cache(k, k)
    table = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 128, 64, dtype=torch.bfloat16, device="cuda")
    call = lambda B, max_len: E.lib().ead_kv_attention(                                              # noqa: E731
        C.byref(cache), C.byref(E.EadKvBatch(B, 1, 1, max_len, table.data_ptr(), table.data_ptr(), table.data_ptr(), 1 << 22, 0)), q.data_ptr(),
        128 * 64, 128, 0.1, 0, 0, q.data_ptr(), 128 * 64, None, workspace.data_ptr(), None, 0, _stream())
    assert call(4096, 1 << 30) == E.EAD_ELIMIT
    assert call(4096, 1 << 24) == E.EAD_ELIMIT


def test_attention_many_sequences(E, workspace):
    rng = np.random.default_rng(12)
    for B, hi in ((700, 40), (4096, 9)):
        length = [int(x) for x in rng.integers(1, hi, B)]
        new = [int(min(l, x)) for l, x in zip(length, rng.integers(0, 12, B))]
        ctx = Context(new, length, 1, 64, 8, seed=12)
        q = _q(ctx, 2)
        _check(_attend(E, ctx, q, workspace, 0.125), attention(ctx, q, 0.125, 0, 0))


def test_attention_reports_bad_pages_and_counts(E, workspace):
    ctx = Context([1, 60], [200, 300], 1, 128, 16, seed=13)
    q = _q(ctx, 4)
    good = _attend(E, ctx, q, workspace, 0.1)
    assert good[2] == 0
    table = ctx.table.copy()
    for bad in (-1, ctx.n_pages, 2 ** 31 - 1):
        for b in (0, 1):
            ctx.table = table.copy()
            ctx.table[b, 3] = bad
            ctx.d_table = torch.from_numpy(ctx.table).cuda()
            got = _attend(E, ctx, q, workspace, 0.1)
            assert got[2] == E.EAD_STATUS_BAD_PAGE, (bad, b)
            other = slice(0, 1) if b == 1 else slice(1, 61)
            assert torch.equal(got[0][other], good[0][other])          # the other sequence is as before
    ctx.d_table = torch.from_numpy(table).cuda()
    assert _attend(E, ctx, q, workspace, 0.1, max_len=256)[2] == E.EAD_STATUS_BAD_PAGE
    got = _attend(E, ctx, q, workspace, 0.1)
    assert got[2] == 0 and torch.equal(got[0], good[0])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,dim,page,layout", [(8, 128, 16, "head"), (1, 64, 8, "head"), (3, 128, 64, "token"), (5, 64, 32, "padded"),
                                                   (128, 64, 16, "head")])
def test_write_and_read(E, fmt, heads, dim, page, layout):
    new, length = [1, 0, 5, 40, 1, 17], [1, 9, 300, 40, 64, 18]
    ctx = Context(new, length, heads, dim, page, fmt, seed=heads, layout=layout, stale=3.0)
    n = int(ctx.new_start[-1])
    g = torch.Generator().manual_seed(2)
    wide = torch.randn(n, 2 * heads + 3, dim, generator=g) * torch.exp(2 * torch.randn(n, 2 * heads + 3, 1, generator=g))
    wide[0, 0, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
    wide[1, :, :32] = 0
    wide[2, :2] *= 2.0 ** 120
    wide[3, :2] *= 2.0 ** -125
    wide = wide.bfloat16()
    dw = wide.cuda()
    before = {k: v.cpu().clone() for k, v in ctx.dev.items()}
    st = _status()
    E.ead_kv_write(ctx.cache(E), ctx.batch(E), dw[:, :heads], dw[:, heads:2 * heads], status=st, stream=_stream())
    assert st.item() == 0
    want_rows = {}
    for name, rows in (("k", wide[:, :heads]), ("v", wide[:, heads:2 * heads])):
        pool, scale = before[name], before.get(name + "_scale")
        codes, by = (rows, None) if fmt == "bf16" else map(torch.from_numpy, quantise(rows.float().numpy()))
        t = 0
        for b, (m, l) in enumerate(zip(new, length)):
            for i in range(m):
                p = l - m + i
                pool[ctx.table[b, p // page], :, p % page] = codes[t]
                if scale is not None:
                    scale[ctx.table[b, p // page], :, p % page] = by[t]
                t += 1
        got = ctx.dev[name].cpu()
        if fmt == "bf16":
            assert torch.equal(got.view(torch.int16), pool.view(torch.int16))
        else:
            assert torch.equal(got, pool) and torch.equal(ctx.dev[name + "_scale"].cpu(), scale)
        want_rows[name] = rows.double() if fmt == "bf16" else torch.from_numpy(values(codes.numpy(), by.numpy()))
    out = torch.full((n, 2 * heads + 1, dim), -7.0, dtype=torch.bfloat16, device="cuda")
    first = torch.tensor([l - m for m, l in zip(new, length)], dtype=torch.int32, device="cuda")
    E.ead_kv_read(ctx.cache(E), ctx.batch(E), out[:, :heads], out[:, heads:2 * heads], first=first, status=st, stream=_stream())
    assert st.item() == 0 and (out[:, 2 * heads:] == -7.0).all()
    for name, o in (("k", out[:, :heads]), ("v", out[:, heads:2 * heads])):
        torch.testing.assert_close(o.cpu().double(), want_rows[name], rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_large_calls_move_what_small_ones_do(E, fmt):
    """One call over 2 * 2051 * 32 * 128 values (more than 2^24) writes and reads bit by bit what a call per sequence does."""
    new, length, heads, dim = [1, 699, 0, 1351], [5, 699, 3, 1400], 32, 128
    whole, apart = (Context(new, length, heads, dim, 16, fmt, seed=7, stale=3.0) for _ in range(2))
    n = int(whole.new_start[-1])
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = torch.randn(n, 2 * heads, dim, generator=g, device="cuda") * torch.exp(torch.randn(n, 2 * heads, 1, generator=g, device="cuda"))
    rows = rows.bfloat16()
    out = torch.empty_like(rows), torch.empty_like(rows)
    first = torch.tensor([l - m for m, l in zip(new, length)], dtype=torch.int32, device="cuda")
    st = _status()
    E.ead_kv_write(whole.cache(E), whole.batch(E), rows[:, :heads], rows[:, heads:], status=st, stream=_stream())
    E.ead_kv_read(whole.cache(E), whole.batch(E), out[0][:, :heads], out[0][:, heads:], first=first, status=st, stream=_stream())
    for b, m in enumerate(new):
        r = slice(int(whole.new_start[b]), int(whole.new_start[b]) + m)
        if m == 0:
            continue
        starts = torch.tensor([0, m], dtype=torch.int32, device="cuda")
        batch = E.ead_kv_batch(apart.d_table[b:b + 1], starts, apart.d_len[b:b + 1], n_tokens=m, max_new=m, max_len=length[b])
        E.ead_kv_write(apart.cache(E), batch, rows[r, :heads], rows[r, heads:], status=st, stream=_stream())
        E.ead_kv_read(apart.cache(E), batch, out[1][r, :heads], out[1][r, heads:], first=first[b:b + 1], status=st, stream=_stream())
    assert st.item() == 0
    for name in whole.dev:
        assert torch.equal(whole.dev[name].view(torch.uint8), apart.dev[name].view(torch.uint8)), name
    assert torch.equal(out[0].view(torch.int16), out[1].view(torch.int16))
    if fmt == "bf16":
        assert torch.equal(out[0], rows)


def test_moves_of_more_than_2_27_tokens(E):
    """The last tokens of a call that passes 2^32 threads are moved like the first ones.  All but the last three positions are
    negative (they have no place), so the cache is small and only the rows are large."""
    n, last = (1 << 27) + 3, 3
    k, v = (torch.full((2, 1, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    cache = E.ead_kv_cache(k, v)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    lens, first = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (last, last - n))
    batch = E.ead_kv_batch(table, starts, lens, n_tokens=n, max_new=n, max_len=16)
    rows = torch.zeros(n, 1, 64, dtype=torch.bfloat16, device="cuda")
    marks = torch.arange(1, 65, dtype=torch.bfloat16, device="cuda") * torch.tensor([1.0, 2.0, -1.0], device="cuda").bfloat16()[:, None]
    rows[-last:, 0] = marks
    st = _status()
    E.ead_kv_write(cache, batch, rows, rows, status=st, stream=_stream())
    assert st.item() == E.EAD_STATUS_BAD_PAGE                          # of the tokens without a place
    for pool in (k, v):
        assert torch.equal(pool[1, 0, :last], marks) and (pool[1, 0, last:] == 3.0).all() and (pool[0] == 3.0).all()
    rows.fill_(9.0)
    E.ead_kv_read(cache, batch, rows, rows, first=first, status=st, stream=_stream())
    assert torch.equal(rows[-last:, 0], marks)
    for at in range(0, n - last, 1 << 24):
        assert not rows[at:min(at + (1 << 24), n - last)].any()
    del rows
    torch.cuda.empty_cache()


def test_every_code_and_scale_reads_exactly(E):
    """All codes under every scale the library writes: bf16 holds each value exactly."""
    codes = torch.arange(256, dtype=torch.uint8)
    codes[codes & 0x7F == 0x7F] = 0
    codes = codes.repeat(240).view(240, 1, 8, 32).repeat(1, 1, 1, 2).contiguous()
    scale = torch.arange(7, 247, dtype=torch.uint8).view(240, 1, 1, 1).repeat(1, 1, 8, 2).contiguous()
    cache = E.ead_kv_cache(codes.cuda(), codes.cuda(), scale.cuda(), scale.cuda())
    table = torch.arange(240, dtype=torch.int32, device="cuda").view(1, 240)
    starts = torch.tensor([0, 1920], dtype=torch.int32, device="cuda")
    k = torch.empty(1920, 1, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    E.ead_kv_read(cache, E.ead_kv_batch(table, starts, n_tokens=1920, max_new=1920, max_len=1920), k, v, stream=_stream())
    want = torch.from_numpy(values(codes.numpy(), scale.numpy())).view(1920, 1, 64)
    torch.testing.assert_close(k.cpu().double(), want, rtol=0, atol=0, equal_nan=True)
    torch.testing.assert_close(v.cpu().double(), want, rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_tokens_without_a_place(E, fmt):
    """Bad pages, negative positions and positions beyond max_len are skipped, read as zeros and reported."""
    ctx = Context([3, 2, 2], [40, 1, 20], 2, 64, 16, fmt, seed=1, stale=3.0)
    ctx.table[0, 2] = ctx.n_pages                                         # positions 32 .. 39 of sequence 0
    ctx.d_table = torch.from_numpy(ctx.table).cuda()
    before = {k: v.cpu().clone() for k, v in ctx.dev.items()}
    rows = torch.ones(7, 2, 64, dtype=torch.bfloat16, device="cuda")
    st = _status()
    E.ead_kv_write(ctx.cache(E), ctx.batch(E, max_len=19), rows, rows, status=st, stream=_stream())
    assert st.item() == E.EAD_STATUS_BAD_PAGE
    changed = (ctx.dev["k"].cpu().view(torch.uint8) != before["k"].view(torch.uint8)).flatten(3).any(3).any(1)    # [page, slot]
    want = torch.zeros_like(changed)
    want[ctx.table[1, 0], 0] = want[ctx.table[2, 1], 2] = True             # sequence 1, token 1 and sequence 2, position 18
    assert torch.equal(changed, want)
    k = torch.full((7, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, 9.0)
    st.zero_()
    E.ead_kv_read(ctx.cache(E), ctx.batch(E, max_len=19), k, v, status=st, stream=_stream(),
                  first=torch.tensor([37, -1, 18], dtype=torch.int32, device="cuda"))
    assert st.item() == E.EAD_STATUS_BAD_PAGE
    zero = (k == 0).flatten(1).all(1).cpu().tolist()
    assert zero == [True, True, True, True, False, False, True]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("case", ["behind", "ahead", "many", "beyond"])
def test_moves_with_counts_that_contradict_each_other(E, fmt, large, case):
    """Tokens behind new_start[B] or before new_start[0], sequences of more than max_new tokens and ones that end behind
    n_tokens: not written, read as zeros, reported, and the other sequences are served.  All of the page table is in range (a
    captured step replays with old entries behind the contexts), so a token that got a place would be seen."""
    heads, dim, page, n = (32, 128, 16, 2100) if large else (2, 64, 16, 12)    # large: more than 2^24 values
    unit = 350 if large else 2
    starts = dict(behind=[0, unit, 2 * unit, 4 * unit], ahead=[unit, 2 * unit, 3 * unit, 6 * unit],
                  many=[0, unit, 5 * unit, 6 * unit], beyond=[0, unit, 3 * unit, 6 * unit + 1])[case]
    served = dict(behind=[0, 1, 2], ahead=[0, 1, 2], many=[0, 2], beyond=[0, 1])[case]
    max_new = 3 * unit + 1
    per = -(-4 * unit // page) + 2
    g = torch.Generator().manual_seed(6)
    table = torch.randperm(3 * per + 4, generator=g)[:3 * per].int().view(3, per)
    lens = torch.tensor([starts[i + 1] - starts[i] + 3 for i in range(3)], dtype=torch.int32)
    shape = (3 * per + 4, heads, page, dim)
    dtype = torch.bfloat16 if fmt == "bf16" else torch.uint8
    k, v = (torch.full(shape, 3, dtype=dtype, device="cuda") for _ in "kv")
    scales = [torch.full((*shape[:3], dim // 32), 120, dtype=torch.uint8, device="cuda") for _ in "kv"] if fmt == "e4m3" else []
    cache = E.ead_kv_cache(k, v, *scales)
    batch = E.ead_kv_batch(table.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda"), lens.cuda(), n_tokens=n, max_new=max_new,
                           max_len=per * page)
    rows = torch.ones(n, heads, dim, dtype=torch.bfloat16, device="cuda")
    st = _status()
    E.ead_kv_write(cache, batch, rows, rows, status=st, stream=_stream())
    assert st.item() == E.EAD_STATUS_BAD_COUNT
    want = torch.zeros(shape[0], page, dtype=torch.bool)
    for b in served:
        for p in range(3, int(lens[b])):
            want[table[b, p // page], p % page] = True
    for pool, old in ((k, 3), (v, 3), *((s, 120) for s in scales)):
        changed = pool != old
        assert torch.equal(changed.any(3).any(1).cpu(), want) and torch.equal(changed.all(3).all(1).cpu(), want)
    out = torch.full((n, 2 * heads, dim), 9.0, dtype=torch.bfloat16, device="cuda")
    st.zero_()
    E.ead_kv_read(cache, batch, out[:, :heads], out[:, heads:], first=torch.full((3,), 3, dtype=torch.int32, device="cuda"), status=st,
                  stream=_stream())
    assert st.item() == E.EAD_STATUS_BAD_COUNT
    ones = torch.zeros(n, dtype=torch.bool)
    for b in served:
        ones[starts[b]:starts[b + 1]] = True
    assert torch.equal((out == 1).flatten(1).all(1).cpu(), ones) and torch.equal((out == 0).flatten(1).all(1).cpu(), ~ones)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,group", [([1, 2, 1], 4), ([40, 70, 30], 4), ([1, 70, 30], 4), ([3, 5, 4], 20)])
def test_attention_reports_counts_that_contradict_each_other(E, workspace, fmt, new, group):
    """Few-rows kernel, chunk kernel and both: sequences of more than max_new tokens or that end behind n_tokens are reported and
    their rows not written; rows behind new_start[B] are not written; the other sequences are as before."""
    ctx = Context(new, [150, 260, 90], 2, 64, 16, fmt, seed=17)
    q = _q(ctx, group)
    good = _attend(E, ctx, q, workspace, 0.1)
    want = attention(ctx, q, 0.1, 0, 0)
    _check(good, want)
    untouched = lambda x, r: bool((x[0][r] == -7.0).all() and (x[1][r] == -7.0).all())          # noqa: E731
    served = lambda x, *rows: [_check((x[0][r], x[1][r], 0), [w[r] for w in want]) for r in rows if len(x[0][r])]   # noqa: E731
    a, b, n = int(ctx.new_start[1]), int(ctx.new_start[2]), int(ctx.new_start[3])
    got = _attend(E, ctx, q, workspace, 0.1, max_new=new[1] - 1) if new[1] * 3 > n + 2 else None
    if got:
        assert got[2] == E.EAD_STATUS_BAD_COUNT and untouched(got, slice(a, b))
        served(got, slice(0, a), slice(b, n))
    got = _attend(E, ctx, q[:n - 1], workspace, 0.1, n_tokens=n - 1)
    assert got[2] == E.EAD_STATUS_BAD_COUNT and untouched(got, slice(b, n - 1))
    served(got, slice(0, b))
    wide = torch.cat([q, q[:1].expand(5, -1, -1)])
    got = _attend(E, ctx, wide, workspace, 0.1, n_tokens=n + 5, max_new=max(new) + 5)
    assert got[2] == 0 and untouched(got, slice(n, n + 5))
    served(got, slice(0, n))
    again = _attend(E, ctx, q, workspace, 0.1)
    assert again[2] == 0 and torch.equal(again[0], good[0]) and torch.equal(again[1], good[1])


@pytest.mark.parametrize("H", [8, 40, 64, 1536, 4096, 5120, 8200, 16384])
@pytest.mark.parametrize("rows,pad,with_residual", [(1, 0, True), (7, 8, True), (300, 0, False)])
def test_norm_bf16(E, H, rows, pad, with_residual):
    g = torch.Generator().manual_seed(H + rows)
    x, r = ((torch.randn(rows, H + pad, generator=g) * torch.exp(torch.randn(H + pad, generator=g))).bfloat16() for _ in range(2))
    w = (1 + 0.3 * torch.randn(H, generator=g)).bfloat16()
    dx, dr = x.cuda(), r.cuda()
    out = torch.full((rows, H + pad), -7.0, dtype=torch.bfloat16, device="cuda")
    E.ead_add_rmsnorm(dx[:, :H], w.cuda(), out[:, :H], residual=dr[:, :H] if with_residual else None,
                      residual_out=dr[:, :H] if with_residual else None, eps=1e-5, stream=_stream())
    s = x[:, :H].double() + (r[:, :H].double() if with_residual else 0)
    y = s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-5) * w.double()
    # one rounding to bf16 (8 significant bits: 2^-8), a 32-bit sum of H squares and a handful of 32-bit roundings (2^-16 covers them)
    assert ((out[:, :H].cpu().double() - y).abs() <= (2.0 ** -8 + 2.0 ** -16) * y.abs() + 1e-30).all()
    assert (out[:, H:] == -7.0).all()
    if with_residual:
        assert torch.equal(dr.cpu()[:, :H], s.float().bfloat16()) and torch.equal(dr.cpu()[:, H:], r[:, H:])
    E.ead_add_rmsnorm(dx[:, :H], w.cuda(), dx[:, :H], eps=1e-5, stream=_stream())      # in place
    s = x[:, :H].double()
    y = s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-5) * w.double()
    assert ((dx[:, :H].cpu().double() - y).abs() <= (2.0 ** -8 + 2.0 ** -16) * y.abs() + 1e-30).all()


@pytest.mark.parametrize("H", [32, 96, 1536, 5120, 8224, 16384])
@pytest.mark.parametrize("rows,pad", [(1, 0), (9, 16)])
def test_norm_e4m3(E, H, rows, pad):
    g = torch.Generator().manual_seed(H + rows)
    x, r = ((torch.randn(rows, H, generator=g) * torch.exp(torch.randn(H, generator=g))).bfloat16() for _ in range(2))
    x[0, :32] = r[0, :32] = 0
    w = (1 + 0.3 * torch.randn(H, generator=g)).bfloat16()
    out = torch.full((rows, H + pad), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.empty(rows, H // 32, dtype=torch.uint8, device="cuda")
    res = torch.empty(rows, H, dtype=torch.bfloat16, device="cuda")
    E.ead_add_rmsnorm(x.cuda(), w.cuda(), out[:, :H], residual=r.cuda(), residual_out=res, out_scale=scale, eps=1e-6, stream=_stream())
    s = x.double() + r.double()
    y = (s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-6) * w.double()).numpy()
    assert torch.equal(res.cpu(), s.float().bfloat16()) and (out[:, H:] == 0x55).all()
    codes, by = quantise(y)
    got_by = scale.cpu().numpy()
    # a block's maximum within 32-bit rounding of a power of two may take the neighbouring scale
    amax = np.abs(y.reshape(rows, -1, 32)).max(-1)
    edge = np.abs(amax / (448.0 * 2.0 ** np.round(np.log2(np.maximum(amax, 1e-300) / 448.0))) - 1) < 2.0 ** -16
    assert (got_by == by)[~edge].all() and (np.abs(got_by.astype(int) - by)[edge] <= 1).all()
    got = values(out[:, :H].cpu().numpy(), got_by)
    step = np.repeat(2.0 ** (got_by.astype(float) - 127), 32, -1)
    # nearest code: half a step of 2^-3 relative (2^-4), or of the subnormal spacing 2^-9 of the scale
    assert (np.abs(got - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * step) * (1 + 2.0 ** -12)).all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,rows", [(64, 30011), (1536, 8111), (4096, 1793), (5120, 2501), (8224, 1903), (16384, 1207)])
@pytest.mark.parametrize("in_place", [False, True])
def test_norm_of_more_rows_than_blocks(E, fmt, H, rows, in_place):
    """Blocks that walk over several rows, the last turn with some of them: every row against the 64-bit result; in place means
    the residual's own buffer for the sum and, for bf16, the input's own for the output."""
    g = torch.Generator(device="cuda").manual_seed(H)
    x, r = ((torch.randn(rows, H, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).bfloat16()
            for _ in range(2))
    w = (1 + 0.3 * torch.randn(H, generator=g, device="cuda")).bfloat16()
    dx, dr = x.clone(), r.clone()
    res = dr if in_place else torch.empty_like(dr)
    if fmt == "bf16":
        out, scale = dx if in_place else torch.empty_like(dx), None
    else:
        out, scale = (torch.empty(rows, n, dtype=torch.uint8, device="cuda") for n in (H, H // 32))
    E.ead_add_rmsnorm(dx, w, out, residual=dr, residual_out=res, out_scale=scale, eps=1e-5, stream=_stream())
    for at in range(0, rows, 1024):
        rows_ = slice(at, at + 1024)
        s = x[rows_].double() + r[rows_].double()
        y = s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-5) * w.double()
        assert torch.equal(res[rows_], s.float().bfloat16())
        if fmt == "bf16":                          # tolerance as for few rows above
            assert ((out[rows_].double() - y).abs() <= (2.0 ** -8 + 2.0 ** -16) * y.abs() + 1e-30).all()
        else:                                      # the smallest power that holds the block, give or take 32-bit rounding; then the nearest code
            power = torch.exp2(scale[rows_].double() - 127)[..., None]
            amax = y.abs().view(len(y), -1, 32).amax(-1, keepdim=True)
            assert (amax <= 448 * power * (1 + 2.0 ** -16)).all() and (amax > 224 * power * (1 - 2.0 ** -16)).all()
            got = (out[rows_].view(torch.float8_e4m3fn).double().view(len(y), -1, 32) * power).view_as(y)
            step = power.expand(-1, -1, 32).reshape(y.shape)
            assert ((got - y).abs() <= torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * step) * (1 + 2.0 ** -12)).all()


@pytest.mark.parametrize("H,rows", [(64, 20000), (5120, 1500)])
def test_norm_writes_the_sum_over_its_input(E, H, rows):
    """residual_out may be x: without a residual that is a copy onto itself, with one the stream's new value."""
    g = torch.Generator(device="cuda").manual_seed(22)
    x, r = (torch.randn(rows, H, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    for residual in (None, r):
        dx, ref, out, res = x.clone(), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        E.ead_add_rmsnorm(x, w, ref, residual=residual, residual_out=res, stream=_stream())
        E.ead_add_rmsnorm(dx, w, out, residual=residual, residual_out=dx, stream=_stream())
        assert torch.equal(out, ref) and torch.equal(dx, res)
        assert torch.equal(res, x if residual is None else (x.float() + r.float()).bfloat16())


def test_norm_of_zeros_and_non_finite_rows(E):
    x = torch.zeros(3, 64, dtype=torch.bfloat16)
    x[1, 5], x[2, 7] = float("inf"), float("nan")
    out = torch.empty(3, 64, dtype=torch.bfloat16, device="cuda")
    E.ead_add_rmsnorm(x.cuda(), torch.ones(64, dtype=torch.bfloat16, device="cuda"), out, eps=1e-6, stream=_stream())
    o = out.cpu()
    assert (o[0] == 0).all() and o[1, 5].isnan() and (o[1, :5] == 0).all() and o[2].isnan().all()


def test_nothing_to_do(E, workspace):
    """A step without new tokens and a norm without rows are no errors (their tensors have no address)."""
    ctx = Context([0, 0], [5, 0], 2, 64, 16, seed=1)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    E.ead_kv_write(ctx.cache(E), ctx.batch(E), none, none, stream=_stream())
    E.ead_kv_read(ctx.cache(E), ctx.batch(E), none, none, stream=_stream())
    E.ead_kv_attention(ctx.cache(E), ctx.batch(E), none, none, scale=1.0, workspace=workspace, stream=_stream())
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    E.ead_add_rmsnorm(x, torch.ones(64, dtype=torch.bfloat16, device="cuda"), x, stream=_stream())
    torch.cuda.synchronize()
