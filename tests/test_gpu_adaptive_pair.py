"""The decoder-side operators and the gate together: the example's generation loop, checked against whole passes."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("e4m3", [False, True])
def test_catching_up_in_chunks_equals_one_pass(e4m3):
    """After generation with switches, every model catches up on every sequence; the hidden states it gets that way
    (token by token, in chunks of the lag, over several calls) match those of one pass over the whole history.

    A one-pass hidden state differs by the order of bf16 roundings only: each of the 3 layers rounds its two
    additions to the stream (relative 2^-8 each, of a stream whose norm the final norm sets to 1 per element), the
    same order as attention's and the matmuls' own roundings: 12 roundings of 2^-8, random in sign."""
    import adaptive_pair as A
    history, log, small, large = A.generate(steps=30, e4m3=e4m3)
    flat = sum(log, [])
    assert 0 < sum(flat) < len(flat)                              # both models produced tokens
    assert any(log[t][b] != log[t - 1][b] for t in range(1, len(log)) for b in range(len(history)))
    everyone = set(range(len(history)))
    for m in (small, large):
        assert any(0 < c < len(h) for c, h in zip(m.cached, history)) or all(c == len(h) - 1 for c, h in zip(m.cached, history))
        late = m.step(history, everyone).float()
        m.forget()
        whole = m.step(history, everyone).float()
        assert m.status.item() == 0
        err = (late - whole).square().mean().sqrt() / whole.square().mean().sqrt()
        assert err < 12 * 2.0 ** -8, err


def test_sliding_window_model_runs_in_the_loop():
    import adaptive_pair as A
    history, log, small, large = A.generate(steps=30, prompt=40, small_kw=dict(window=16, sinks=2))
    assert small.status.item() == 0 and large.status.item() == 0
    everyone = set(range(len(history)))
    late = small.step(history, everyone).float()
    small.forget()
    whole = small.step(history, everyone).float()
    err = (late - whole).square().mean().sqrt() / whole.square().mean().sqrt()
    assert err < 12 * 2.0 ** -8, err
