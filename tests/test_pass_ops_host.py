"""CPU-only checks of the operators of a decoder's 8-bit pass: argument validation before anything touches a GPU, the binding's own
checks, and the test suite's block quantisation against torch's conversion."""
import ctypes as C

import numpy as np
import pytest
import torch

import pass_util as P


@pytest.fixture(scope="module")
def E():
    from paper_2502_06833_b200 import build
    build.build()
    from paper_2502_06833_b200 import binding
    return binding


def _code(E, letter):
    return dict(I=E.EAD_EINVALID_ARG, A=E.EAD_EALIGNMENT, L=E.EAD_ELIMIT, O=E.EAD_OK)[letter]


def _matrix(E, rows=4, cols=64, block_rows=1, block_cols=32, row_stride=64, codes=4096, scale=4096, reserved=0):
    return E.EadE4m3Matrix(rows, cols, block_rows, block_cols, row_stride, codes, scale, reserved)


def _linear(E, x=None, w=None, bias=None, format=0, out=8192, out_stride=128, status=None):
    x = _matrix(E) if x is None else x
    w = _matrix(E, rows=128, block_rows=128, block_cols=128) if w is None else w
    ref = lambda m: None if m == 0 else C.byref(m)                       # noqa: E731
    return E.lib().ead_linear(ref(x), ref(w), bias, format, out, out_stride, status, 0, None)


BAD_MATRIX = [(dict(rows=-1), "I"), (dict(rows=(1 << 30) + 1), "I"), (dict(cols=0), "I"), (dict(cols=16), "I"), (dict(cols=72, row_stride=80), "A"),
              (dict(row_stride=48), "I"), (dict(row_stride=72), "A"), (dict(row_stride=1 << 40), "I"), (dict(codes=None), "I"), (dict(codes=4104), "A"),
              (dict(scale=None), "I"), (dict(scale=4098), "A"), (dict(reserved=1), "I"), (dict(block_rows=2), "I"), (dict(block_cols=64), "I"),
              (dict(block_rows=128), "I")]


@pytest.mark.parametrize("bad,letter", BAD_MATRIX)
def test_bad_matrices_are_refused(E, bad, letter):
    assert _linear(E, x=_matrix(E, **bad)) == _code(E, letter)
    if "block_rows" not in bad or bad["block_rows"] == 2:
        assert E.lib().ead_quantise(4096, 64, None, 0, C.byref(_matrix(E, **bad)), 0, None) == _code(E, letter)
    if not ({"block_cols", "block_rows"} & set(bad)) and bad != dict(scale=4098):
        assert _linear(E, w=_matrix(E, **{**dict(rows=128, block_rows=128, block_cols=128), **bad})) == _code(E, letter)


@pytest.mark.parametrize("bad,letter", [
    (dict(x=0), "I"), (dict(w=0), "I"), (dict(format=1), "I"), (dict(format=3), "I"), (dict(out=None), "I"), (dict(out=8193), "A"),
    (dict(out_stride=127), "I"), (dict(out=8194, format=2), "A"), (dict(status=4098), "A"), (dict(bias=4097), "A")])
def test_bad_products_are_refused(E, bad, letter):
    assert _linear(E, **bad) == _code(E, letter)


def test_products_of_unlike_operands_are_refused(E):
    bad = _code(E, "I")
    assert _linear(E, x=_matrix(E, cols=96, row_stride=96)) == bad
    assert _linear(E, x=_matrix(E, block_rows=128, block_cols=128)) == bad
    assert _linear(E, w=_matrix(E, rows=128)) == bad and _linear(E, w=_matrix(E, rows=128, block_cols=128)) == bad
    tall = _matrix(E, rows=1 << 30), _matrix(E, rows=1 << 30, block_rows=128, block_cols=128)
    assert _linear(E, *tall, out_stride=1 << 30) == _code(E, "L")
    # nothing to do: rows without an address
    assert _linear(E, x=_matrix(E, rows=0, codes=None, scale=None), out=None) == E.EAD_OK
    assert _linear(E, w=_matrix(E, rows=0, codes=None, scale=None, block_rows=128, block_cols=128), out=None) == E.EAD_OK


@pytest.mark.parametrize("args,letter", [
    ((None, 64, None, 0), "I"), ((4100, 64, None, 0), "A"), ((4096, 56, None, 0), "I"), ((4096, 68, None, 0), "A"), ((4096, 64, 4100, 64), "A"),
    ((4096, 64, 4096, 8), "I"), ((4096, 64, 4096, 68), "A")])
def test_bad_rows_to_quantise_are_refused(E, args, letter):
    assert E.lib().ead_quantise(*args, C.byref(_matrix(E)), 0, None) == _code(E, letter)
    assert E.lib().ead_quantise(*args, None, 0, None) == E.EAD_EINVALID_ARG


def test_quantise_limits(E):
    q = E.lib().ead_quantise
    assert q(4096, 64, 4096, 64, C.byref(_matrix(E, block_rows=128, block_cols=128)), 0, None) == E.EAD_EINVALID_ARG      # a gate and tiles
    assert q(None, 64, None, 0, C.byref(_matrix(E, rows=0, codes=None, scale=None)), 0, None) == E.EAD_OK


def _rope(E, head_dim=64, rot_dim=64, interleaved=0, eps=1e-6, inv_freq=4096, q_weight=4096, k_weight=4096, reserved=0):
    return E.EadRope(head_dim, rot_dim, interleaved, eps, inv_freq, q_weight, k_weight, reserved)


def _kv(E, **kw):
    c = E.EadKvCache(0, 2, 64, 16, 4, 0, 2048, 1024, 64, 4096, 8192, None, None)
    b = E.EadKvBatch(3, 5, 4, 60, 4096, 4096, 4096, 4, 0)
    for k, v in kw.items():
        setattr(c if hasattr(c, k) else b, k, v)
    return c, b


DENSE = dict(positions=4096, n=3, q=4096, q_stride=512, heads_q=8, k=4096, k_stride=128, heads_kv=2, q_out=8192, qo_stride=512, k_out=8192, ko_stride=128)
PAGED = dict(positions=None, q=4096, q_stride=512, heads_q=8, k=4096, v=4096, kv_stride=128, q_out=8192, qo_stride=512, status=None)


def _dense(E, rope, **kw):
    return E.lib().ead_qk_norm_rope(rope and C.byref(rope), *{**DENSE, **kw}.values(), 0, None)


def _paged(E, rope, kv=None, **kw):
    c, b = kv or _kv(E)
    return E.lib().ead_kv_rotate_write(rope and C.byref(rope), C.byref(c), C.byref(b), *{**PAGED, **kw}.values(), 0, None)


@pytest.mark.parametrize("bad,letter", [
    (dict(head_dim=96), "I"), (dict(head_dim=256), "I"), (dict(rot_dim=-16), "I"), (dict(rot_dim=80), "I"), (dict(rot_dim=24), "I"), (dict(interleaved=2), "I"),
    (dict(eps=-1.0), "I"), (dict(eps=float("nan")), "I"), (dict(eps=float("inf")), "I"), (dict(inv_freq=None), "I"), (dict(inv_freq=4098), "A"),
    (dict(q_weight=4104), "A"), (dict(k_weight=4100), "A"), (dict(reserved=1), "I")])
def test_bad_ropes_are_refused(E, bad, letter):
    assert _dense(E, _rope(E, **bad)) == _code(E, letter)
    assert _paged(E, _rope(E, **bad)) == _code(E, letter)


def test_no_rope_is_refused(E):
    assert _dense(E, None) == E.EAD_EINVALID_ARG and _paged(E, None) == E.EAD_EINVALID_ARG


@pytest.mark.parametrize("bad,letter", [
    (dict(positions=None), "I"), (dict(positions=4098), "A"), (dict(n=-1), "I"), (dict(n=(1 << 30) + 1), "I"), (dict(n=0, positions=None), "O"),
    (dict(q=None), "I"), (dict(q=4100), "A"), (dict(q_stride=504), "I"), (dict(q_stride=516), "A"), (dict(heads_q=-1), "I"), (dict(heads_q=16385), "I"),
    (dict(heads_kv=129), "I"), (dict(heads_kv=-1), "I"), (dict(k=None), "I"), (dict(k_stride=120), "I"), (dict(q_out=None), "I"), (dict(q_out=8200), "A"),
    (dict(qo_stride=8), "I"), (dict(k_out=None), "I"), (dict(ko_stride=132), "A"), (dict(heads_q=0, heads_kv=0, positions=None), "O")])
def test_bad_heads_are_refused(E, bad, letter):
    assert _dense(E, _rope(E), **bad) == _code(E, letter)


@pytest.mark.parametrize("bad,letter", [
    (dict(positions=4098), "A"), (dict(q=None), "I"), (dict(q=4100), "A"), (dict(q_stride=504), "I"), (dict(heads_q=-1), "I"), (dict(heads_q=16385), "I"),
    (dict(k=None), "I"), (dict(k=4100), "A"), (dict(v=None), "I"), (dict(v=4104), "A"), (dict(kv_stride=120), "I"), (dict(kv_stride=132), "A"),
    (dict(q_out=None), "I"), (dict(q_out=8200), "A"), (dict(qo_stride=100), "I"), (dict(status=4097), "A")])
def test_bad_rotating_writes_are_refused(E, bad, letter):
    assert _paged(E, _rope(E), **bad) == _code(E, letter)


def test_rotating_writes_check_cache_and_batch(E):
    assert _paged(E, _rope(E, head_dim=128)) == E.EAD_EINVALID_ARG       # the cache's heads have 64
    for bad, letter in ((dict(page_size=48), "I"), (dict(heads_kv=0), "I"), (dict(slot_stride=68), "A"), (dict(B=0), "I"), (dict(max_new=1), "I"),
                        (dict(kv_len=None), "I"), (dict(new_start=4098), "A"), (dict(table_stride=0), "I"), (dict(n_tokens=0), "O")):
        assert _paged(E, _rope(E), _kv(E, **bad)) == _code(E, letter), bad


@pytest.mark.parametrize("bad,letter", [
    (dict(logits=None), "I"), (dict(logits=4097), "A"), (dict(format=1), "I"), (dict(format=4), "I"), (dict(format=2, logits=4098), "A"), (dict(stride=99), "I"),
    (dict(n=-1), "I"), (dict(n=0, logits=None), "O"), (dict(V=0), "I"), (dict(V=(1 << 30) + 1, stride=1 << 31), "I"), (dict(tokens=None), "I"),
    (dict(tokens=4098), "A"), (dict(logprob=4098), "A"), (dict(entropy=4097), "A"), (dict(rank=4097), "A"), (dict(k=-1), "I"), (dict(k=65), "L"),
    (dict(top=4098), "A"), (dict(top_logprob=4098), "A"), (dict(workspace=None), "I"), (dict(workspace=4224), "A"), (dict(status=4098), "A")])
def test_bad_scores_are_refused(E, bad, letter):
    a = {**dict(logits=4096, format=0, stride=100, n=2, V=100, tokens=4096, logprob=4096, entropy=4096, rank=4096, k=5, top=4096, top_logprob=4096,
                workspace=4096, status=None), **bad}
    assert E.lib().ead_token_logprobs(*a.values(), 0, None) == _code(E, letter)


def test_binding_refuses_wrong_types_and_shapes(E):
    b8, u8 = (lambda *s: torch.zeros(*s, dtype=torch.uint8)), torch.uint8
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)                # noqa: E731
    x, w = E.ead_e4m3_matrix(b8(3, 160), b8(3, 5), block=(1, 32)), E.ead_e4m3_matrix(b8(130, 160), b8(2, 2), block=(128, 128))
    assert (x.row_stride, w.rows, w.block_cols) == (160, 130, 128)
    assert E.ead_e4m3_matrix(b8(3, 192)[:, :160].view(torch.float8_e4m3fn), b8(3, 2), block=(1, 128)).row_stride == 192
    space, small = torch.zeros(E.EAD_LOGPROB_WORKSPACE_BYTES, dtype=u8), torch.zeros(16, dtype=u8)
    rope = E.ead_rope(torch.zeros(32), 64, q_weight=bf(64))
    assert (rope.rot_dim, rope.head_dim) == (64, 64)
    cache = E.ead_kv_cache(bf(4, 2, 16, 64), bf(4, 2, 16, 64))
    batch = E.ead_kv_batch(torch.zeros(1, 4, dtype=torch.int32), torch.tensor([0, 2], dtype=torch.int32), torch.tensor([9], dtype=torch.int32),
                           n_tokens=2, max_new=2, max_len=9)
    place = torch.zeros(2, dtype=torch.int32)
    q, k = bf(2, 8, 64), bf(2, 2, 64)
    for bad in (lambda: E.ead_e4m3_matrix(b8(3, 160), b8(3, 4), block=(1, 32)), lambda: E.ead_e4m3_matrix(b8(3, 160), b8(3, 5), block=(1, 64)),
                lambda: E.ead_e4m3_matrix(b8(3, 160), b8(3, 5).int(), block=(1, 32)), lambda: E.ead_e4m3_matrix(b8(160, 3).t(), b8(3, 5), block=(1, 32)),
                lambda: E.ead_e4m3_matrix(bf(3, 160), b8(3, 5), block=(1, 32)),
                lambda: E.ead_quantise(bf(3, 128), x), lambda: E.ead_quantise(bf(3, 160).float(), x), lambda: E.ead_quantise(bf(3, 160), x, gate=bf(2, 160)),
                lambda: E.ead_linear(x, w, bf(3, 128)), lambda: E.ead_linear(x, w, bf(3, 130).half()),
                lambda: E.ead_linear(x, w, bf(3, 136)[:, :130], bias=bf(128)), lambda: E.ead_linear(x, w, bf(3, 136)[:, :130], bias=torch.zeros(130)),
                lambda: E.ead_rope(torch.zeros(32).double(), 64), lambda: E.ead_rope(torch.zeros(32), 64, q_weight=bf(32)),
                lambda: E.ead_rope(torch.zeros(32), 64, k_weight=torch.zeros(64)),
                lambda: E.ead_qk_norm_rope(rope, place.long(), q, k, q, k), lambda: E.ead_qk_norm_rope(rope, place, q[:1], k, q, k),
                lambda: E.ead_qk_norm_rope(rope, place, q, k, q[:, :4], k), lambda: E.ead_qk_norm_rope(rope, place, q, k.float(), q, k),
                lambda: E.ead_qk_norm_rope(rope, place, q, bf(2, 2, 32), q, k),
                lambda: E.ead_kv_rotate_write(rope, cache, batch, q, k, bf(2, 4, 64)[:, :2], q), lambda: E.ead_kv_rotate_write(rope, cache, batch, q, bf(2, 1, 64), k, q),
                lambda: E.ead_kv_rotate_write(rope, cache, batch, q, k, k, q[:, :2]), lambda: E.ead_kv_rotate_write(rope, cache, batch, q, k, k, q, positions=place[:1]),
                lambda: E.ead_token_logprobs(torch.zeros(2, 9).double(), place, workspace=space), lambda: E.ead_token_logprobs(torch.zeros(2, 9), place.long(), workspace=space),
                lambda: E.ead_token_logprobs(torch.zeros(2, 9), place[:1], workspace=space), lambda: E.ead_token_logprobs(torch.zeros(2, 9), place, workspace=small),
                lambda: E.ead_token_logprobs(torch.zeros(2, 9), place, logprob=torch.zeros(3), workspace=space),
                lambda: E.ead_token_logprobs(torch.zeros(2, 9), place, top=torch.zeros(2, 3), workspace=space),
                lambda: E.ead_token_logprobs(torch.zeros(2, 9), place, top=torch.zeros(2, 3, dtype=torch.int32), top_logprob=torch.zeros(2, 4), workspace=space),
                lambda: E.ead_token_logprobs(torch.zeros(9, 2).t(), place, workspace=space)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("block,block_rows", [(32, 1), (128, 1), (128, 128)])
def test_block_quantisation_agrees_with_torch(block, block_rows):
    x = np.random.default_rng(0).normal(0, 1, (200, 352)).astype(np.float32)
    x[0, :3] = [0.0, 1e-30, 3e4]
    c, s = P.quantise(x, block, block_rows)
    assert s.shape == (P.up(200, block_rows), P.up(352, block))
    step = np.repeat(np.repeat(2.0 ** (s.astype(np.float64) - 127), block_rows, 0)[:200], block, 1)[:, :352]
    assert np.array_equal(torch.from_numpy((x / step).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), c)
    top = np.abs(x)
    assert (top <= 448 * step).all()
    v = P.values(c, s, block, block_rows)
    assert (np.abs(v - x) <= np.maximum(2.0 ** -4 * top, 2.0 ** -10 * step)).all()
