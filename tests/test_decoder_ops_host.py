"""CPU-only checks of the decoder-side operators: argument validation before anything touches a GPU, the
binding's own checks, and the test suite's 8-bit arithmetic against torch's conversion."""
import numpy as np
import pytest
import torch

from decoder_util import e4m3_grid, quantise, values


@pytest.fixture(scope="module")
def E():
    from paper_2502_06833_b200 import build
    build.build()
    from paper_2502_06833_b200 import binding
    return binding


def _cache(E, **kw):
    c = E.EadKvCache(0, 2, 64, 16, 4, 0, 2048, 1024, 64, 4096, 8192, None, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _batch(E, **kw):
    b = E.EadKvBatch(3, 5, 4, 60, 4096, 4096, 4096, 4, 0)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


BAD_CACHE = [(dict(format=2), "I"), (dict(heads_kv=0), "I"), (dict(heads_kv=129), "I"), (dict(head_dim=96), "I"),
             (dict(page_size=4), "I"), (dict(page_size=48), "I"), (dict(page_size=512), "I"), (dict(n_pages=0), "I"),
             (dict(k=None), "I"), (dict(v=None), "I"), (dict(reserved=1), "I"), (dict(slot_stride=32), "I"),
             (dict(head_stride=-8), "I"), (dict(page_stride=-8), "I"), (dict(k_scale=4096), "I"),
             (dict(format=1), "I"), (dict(format=1, k_scale=4096), "I"), (dict(k=4104), "A"), (dict(v=8200), "A"),
             (dict(slot_stride=68), "A"), (dict(head_stride=1028), "A"), (dict(page_stride=2052), "A"),
             (dict(format=1, k_scale=4096, v_scale=4096, slot_stride=72), "A"),
             (dict(format=1, k_scale=4097, v_scale=4096), "A")]
BAD_BATCH = [(dict(B=0), "I"), (dict(B=4097), "I"), (dict(n_tokens=-1), "I"), (dict(max_new=-1), "I"),
             (dict(max_new=1), "I"), (dict(max_len=-1), "I"), (dict(max_len=65), "I"), (dict(new_start=None), "I"),
             (dict(page_table=None), "I"), (dict(table_stride=0), "I"), (dict(reserved=3), "I"),
             (dict(new_start=4098), "A"), (dict(page_table=4097), "A"),
             (dict(max_len=(1 << 30) + 1, table_stride=1 << 28), "I"),
             (dict(n_tokens=(1 << 30) + 1, max_new=1 << 30), "I")]


def _code(E, letter):
    return dict(I=E.EAD_EINVALID_ARG, A=E.EAD_EALIGNMENT, L=E.EAD_ELIMIT)[letter]


def _calls(E, cache, batch):
    import ctypes as C
    L, c, b = E.lib(), C.byref(cache), C.byref(batch)
    return [L.ead_kv_write(c, b, 4096, 8192, 128, None, 0, None), L.ead_kv_read(c, b, None, 4096, 8192, 128, None, 0, None),
            L.ead_kv_attention(c, b, 4096, 512, 8, 0.1, 0, 0, 8192, 512, None, 4096, None, 0, None)]


@pytest.mark.parametrize("bad,letter", BAD_CACHE)
def test_bad_caches_are_refused(E, bad, letter):
    assert _calls(E, _cache(E, **bad), _batch(E)) == [_code(E, letter)] * 3


@pytest.mark.parametrize("bad,letter", BAD_BATCH)
def test_bad_batches_are_refused(E, bad, letter):
    assert _calls(E, _cache(E), _batch(E, **bad)) == [_code(E, letter)] * 3


def test_null_descriptions_are_refused(E):
    import ctypes as C
    L, c, b = E.lib(), C.byref(_cache(E)), C.byref(_batch(E))
    for x, y in ((None, b), (c, None)):
        assert L.ead_kv_write(x, y, 4096, 8192, 128, None, 0, None) == E.EAD_EINVALID_ARG
        assert L.ead_kv_read(x, y, None, 4096, 8192, 128, None, 0, None) == E.EAD_EINVALID_ARG
        assert L.ead_kv_attention(x, y, 4096, 512, 8, 0.1, 0, 0, 8192, 512, None, 4096, None, 0, None) == E.EAD_EINVALID_ARG
    no_len = C.byref(_batch(E, kv_len=None))
    assert L.ead_kv_write(c, no_len, 4096, 8192, 128, None, 0, None) == E.EAD_EINVALID_ARG
    assert L.ead_kv_attention(c, no_len, 4096, 512, 8, 0.1, 0, 0, 8192, 512, None, 4096, None, 0, None) == E.EAD_EINVALID_ARG


@pytest.mark.parametrize("args,letter", [
    ((None, 8192, 128), "I"), ((4096, None, 128), "I"), ((4096, 8192, 120), "I"), ((4096, 8192, 132), "A"),
    ((4100, 8192, 128), "A"), ((4096, 8196, 128), "A")])
def test_bad_rows_are_refused(E, args, letter):
    import ctypes as C
    L, c, b = E.lib(), C.byref(_cache(E)), C.byref(_batch(E))
    assert L.ead_kv_write(c, b, *args, None, 0, None) == _code(E, letter)
    assert L.ead_kv_read(c, b, None, *args, None, 0, None) == _code(E, letter)
    assert L.ead_kv_write(c, b, 4096, 8192, 128, 4098, 0, None) == E.EAD_EALIGNMENT
    assert L.ead_kv_read(c, b, 4098, 4096, 8192, 128, None, 0, None) == E.EAD_EALIGNMENT


@pytest.mark.parametrize("bad,letter", [
    (dict(q=None), "I"), (dict(q=4100), "A"), (dict(q_stride=504), "I"), (dict(q_stride=516), "A"), (dict(heads_q=1), "I"),
    (dict(heads_q=7), "I"), (dict(heads_q=258, q_stride=258 * 64), "I"), (dict(scale=0.0), "I"), (dict(scale=-1.0), "I"),
    (dict(scale=float("nan")), "I"), (dict(scale=float("inf")), "I"), (dict(window=-1), "I"), (dict(sinks=-1), "I"),
    (dict(out=None), "I"), (dict(out=8200), "A"), (dict(out_stride=100), "I"), (dict(lse=4098), "A"), (dict(workspace=None), "I"),
    (dict(workspace=4096 + 128), "A"), (dict(status=4097), "A")])
def test_bad_attention_arguments_are_refused(E, bad, letter):
    import ctypes as C
    a = {**dict(q=4096, q_stride=512, heads_q=8, scale=0.1, window=0, sinks=0, out=8192, out_stride=512, lse=None, workspace=4096,
                status=None), **bad}
    assert E.lib().ead_kv_attention(C.byref(_cache(E)), C.byref(_batch(E)), *a.values(), 0, None) == _code(E, letter)


@pytest.mark.parametrize("bad,letter", [
    (dict(x=None), "I"), (dict(x=4100), "A"), (dict(x_stride=56), "I"), (dict(x_stride=68), "A"), (dict(residual=4100), "A"),
    (dict(residual_stride=8), "I"), (dict(residual_out=4100), "A"), (dict(weight=None), "I"), (dict(weight=4104), "A"),
    (dict(eps=-1.0), "I"), (dict(eps=float("nan")), "I"), (dict(n=-1), "I"), (dict(H=4), "I"), (dict(H=60), "A"),
    (dict(H=16392, x_stride=16392), "L"), (dict(format=2), "I"), (dict(format=1), "I"), (dict(out_scale=4096), "I"),
    (dict(format=1, out_scale=4096, H=40), "A"), (dict(out=None), "I"), (dict(out=4100), "A"), (dict(out_stride=32), "I")])
def test_bad_norm_arguments_are_refused(E, bad, letter):
    a = {**dict(x=4096, x_stride=64, residual=4096, residual_stride=64, residual_out=4096, residual_out_stride=64, weight=4096,
                eps=1e-6, n=2, H=64, format=0, out=8192, out_stride=64, out_scale=None), **bad}
    assert E.lib().ead_add_rmsnorm(*a.values(), 0, None) == _code(E, letter)


def test_binding_refuses_wrong_types_and_shapes(E):
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, starts, lens = torch.zeros(1, 4, dtype=torch.int32), torch.tensor([0, 2], dtype=torch.int32), torch.tensor([9], dtype=torch.int32)
    for bad in (lambda: E.ead_kv_cache(k.float(), k), lambda: E.ead_kv_cache(k, k[:3]), lambda: E.ead_kv_cache(k[0], k[0]),
                lambda: E.ead_kv_cache(k, k, torch.zeros(4, 2, 16, 2, dtype=torch.uint8)),
                lambda: E.ead_kv_cache(k.byte(), k.byte(), torch.zeros(4, 2, 16, 2, dtype=torch.uint8)),
                lambda: E.ead_kv_cache(k.byte(), k.byte(), *[torch.zeros(4, 2, 16, 4, dtype=torch.uint8)] * 2),
                lambda: E.ead_kv_cache(k.transpose(2, 3), k.transpose(2, 3)),
                lambda: E.ead_kv_batch(table.long(), starts, lens, n_tokens=2, max_new=2, max_len=9),
                lambda: E.ead_kv_batch(table, starts[:1], lens, n_tokens=2, max_new=2, max_len=9),
                lambda: E.ead_kv_batch(table, starts, lens[:0], n_tokens=2, max_new=2, max_len=9)):
        with pytest.raises(ValueError):
            bad()
    cache, batch = E.ead_kv_cache(k, k), E.ead_kv_batch(table, starts, lens, n_tokens=2, max_new=2, max_len=9)
    new, q, ws = torch.zeros(2, 2, 64).bfloat16(), torch.zeros(2, 8, 64).bfloat16(), torch.zeros(16, dtype=torch.uint8)
    for bad in (lambda: E.ead_kv_write(cache, batch, new.float(), new), lambda: E.ead_kv_write(cache, batch, new[:1], new),
                lambda: E.ead_kv_write(cache, batch, new, torch.zeros(2, 4, 64).bfloat16()[:, :2]),
                lambda: E.ead_kv_read(cache, batch, new, new.float()),
                lambda: E.ead_kv_read(cache, batch, new, new, first=torch.zeros(2, dtype=torch.int32)),
                lambda: E.ead_kv_attention(cache, batch, q, q, scale=1.0, workspace=ws),
                lambda: E.ead_kv_attention(cache, batch, q.float(), q, scale=1.0, workspace=ws),
                lambda: E.ead_kv_attention(cache, batch, q, q[:, :4], scale=1.0, workspace=ws),
                lambda: E.ead_kv_attention(cache, batch, q, q, scale=1.0, workspace=ws, lse=torch.zeros(2, 4)),
                lambda: E.ead_add_rmsnorm(q[:, 0], torch.zeros(32).bfloat16(), q[:, 0]),
                lambda: E.ead_add_rmsnorm(q[:, 0], torch.zeros(64).bfloat16(), q[:, 0].float()),
                lambda: E.ead_add_rmsnorm(q[:, 0], torch.zeros(64).bfloat16(), q[:, 0], residual=q[:1, 0]),
                lambda: E.ead_add_rmsnorm(q[:, 0], torch.zeros(64).bfloat16(), q[:, 0].byte(), out_scale=torch.zeros(2, 3, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            bad()


def test_strides_of_dimensions_of_one_element_do_not_matter(E):
    """torch gives a dimension of one element any stride; it addresses nothing."""
    pools = torch.zeros(4, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 16, 64, dtype=torch.bfloat16)
    odd = [x.as_strided((4, 1, 16, 64), (1024, s, 64, 1)) for x, s in zip(pools, (3, 1024))]
    cache = E.ead_kv_cache(*odd)
    assert (cache.page_stride, cache.slot_stride) == (1024, 64) and cache.head_stride % 8 == 0 and cache.heads_kv == 1
    one = torch.zeros(2, 16, 64, dtype=torch.bfloat16)
    odd = [one.as_strided((1, 2, 16, 64), (s, 1024, 64, 1)) for s in (5, 2048)]
    cache = E.ead_kv_cache(*odd)
    assert cache.page_stride % 8 == 0 and (cache.head_stride, cache.n_pages) == (1024, 1)
    with pytest.raises(ValueError):                # others do matter
        E.ead_kv_cache(torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 16, 2, 64).bfloat16().transpose(1, 2))
    starts, lens = torch.tensor([0, 1, 2], dtype=torch.int32), torch.tensor([9, 9], dtype=torch.int32)
    batch = E.ead_kv_batch(torch.zeros(1, 2, dtype=torch.int32).t(), starts, lens, n_tokens=2, max_new=1, max_len=16)
    assert batch.table_stride == 1
    batch = E.ead_kv_batch(torch.zeros(1, 0, dtype=torch.int32), starts[:2], lens[:1], n_tokens=1, max_new=1, max_len=0)
    assert batch.table_stride == 1                 # contexts that have no page yet


def test_grid_and_rounding_agree_with_torch():
    g = e4m3_grid()
    assert len(g) == 127 and g[-1] == 448 and (np.diff(g) > 0).all()
    codes = torch.arange(127, dtype=torch.uint8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).float().numpy(), g)
    x = np.random.default_rng(0).normal(0, 1, (64, 128)).astype(np.float32)
    x[0, :4] = [0.0, -0.0, 1e-30, 3e38]
    c, s = quantise(x)
    scaled = x / 2.0 ** np.repeat(s.astype(np.float64) - 127, 32, -1)
    scaled = np.clip(scaled, -448, 448)             # only the block at the largest scale reaches beyond
    assert np.array_equal(torch.from_numpy(scaled).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy(), c)
    amax = np.abs(x.reshape(64, -1, 32)).max(-1).astype(np.float64)
    assert ((amax <= 448 * 2.0 ** (s.astype(float) - 127)) | (s == 246)).all() and (amax > 448 * 2.0 ** (s.astype(float) - 128)).all()
    assert np.abs(values(c, s) - np.clip(x, -448 * 2.0 ** 119, 448 * 2.0 ** 119)).max() <= 2.0 ** -4 * np.abs(x).max()


def _chunk_plan(n, kv, group, window=0, sinks=0):
    """Units of two row tiles of whole tokens, each 12 + (2 | 1) per tile of 64 keys some query of it sees: tiles of the
    sinks and of the window, none twice, at least one.  Vectorised over the units, in Python integers at the end."""
    per = 128 // group
    i0 = np.arange(0, n, 2 * per, dtype=np.int64)
    tokens = np.minimum(2 * per, n - i0)
    pa = kv - n + i0
    hi = np.clip(pa + tokens, 0, kv)
    lo = np.minimum(np.maximum(pa - window + 1, 0), hi) if window else np.zeros_like(hi)
    first = lo // 64
    sink_tiles = np.minimum(-(-np.minimum(sinks, lo) // 64), first)
    tiles = np.maximum(1, sink_tiles - (-hi // 64) - first)
    return len(i0), sum((12 + np.where(tokens > per, 2, 1) * tiles).tolist())


@pytest.mark.parametrize("n,kv,group", [(525000, 525000, 128), (1050000, 1050000, 32), (2200000, 2200000, 8), (3100000, 3100000, 4),
                                        (300000, 10300000, 8), (1500000, 1 << 30, 16), (1000000, 1 << 30, 128)])
def test_chunk_costs_of_the_longest_prompts(E, n, kv, group):
    """The work string of the chunk kernel passes 32 bits for prompts that the entry point takes."""
    units, cost = _chunk_plan(n, kv, group)
    assert cost > 2 ** 31
    assert E.ead_plan_chunk(n, kv, heads_per_kv=group) == dict(units=units, cost=cost)


@pytest.mark.parametrize("group", [1, 4, 5, 16, 71, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (100, 4), (1024, 65), (200, 300), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_chunk_costs_of_ordinary_chunks(E, group, window, sinks):
    for n, kv in ((17, 17), (40, 900), (200, 150), (2041, 8000), (1, 5)):
        want = _chunk_plan(n, kv, group, window, sinks if window else 0) if n * group > 16 else (0, 0)
        assert E.ead_plan_chunk(n, kv, heads_per_kv=group, window=window, sinks=sinks) == dict(units=want[0], cost=want[1]), (n, kv)
    assert E.ead_plan_chunk(2, 50, heads_per_kv=4, max_new=200)["units"] == 0 and E.ead_plan_chunk(3, 50, heads_per_kv=4, max_new=200)["units"] == 1
    for bad in (dict(n_new=-1), dict(n_new=9, max_new=8), dict(kv_len=-1), dict(kv_len=(1 << 30) + 1), dict(heads_per_kv=0),
                dict(heads_per_kv=129), dict(window=-1), dict(sinks=-1), dict(n_new=1 << 24, heads_per_kv=128)):
        with pytest.raises(E.EadError) as err:
            E.ead_plan_chunk(**{**dict(n_new=4, kv_len=50, heads_per_kv=4), **bad})
        assert err.value.code == E.EAD_EINVALID_ARG
