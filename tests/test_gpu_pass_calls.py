"""Ways to call the operators of a decoder's 8-bit pass: captured as a whole with copies between, in branches of one graph, on two streams at once,
with nothing to do, and without queries."""
import pytest
import torch

import pass_util as P
from decoder_util import Context

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    from paper_2502_06833_b200 import binding
    return binding


def _matrix(E, rows, cols, block):
    return E.ead_e4m3_matrix(torch.zeros(rows, cols, dtype=torch.uint8, device="cuda"),
                             torch.zeros(P.up(rows, block[0]), P.up(cols, block[1]), dtype=torch.uint8, device="cuda"), block=block)


class Chain:
    """Rotation in place, gated quantisation, a product and log probabilities of its rows, on buffers of its own."""

    def __init__(self, E, T, K, V, seed):
        self.E, self.T, self.K, self.V = E, T, K, V
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()          # noqa: E731
        self.inputs = [(rnd(T, K), rnd(T, K), torch.randint(0, V, (T,), generator=g, device="cuda").int()) for _ in range(4)]
        self.x, self.gate, self.token = (torch.empty_like(t) for t in self.inputs[0])
        self.w, self.q = _matrix(E, V, K, (128, 128)), _matrix(E, T, K, (1, 128))
        E.ead_quantise(rnd(V, K), self.w, stream=E.current_stream())
        self.logits, self.space = torch.empty(T, V, device="cuda"), torch.zeros(E.EAD_LOGPROB_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
        self.rope = E.ead_rope((10000.0 ** -(torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().cuda(), 64)
        self.place = torch.arange(T, dtype=torch.int32, device="cuda")
        self.lp, self.rank = torch.empty(T, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda")
        self.top, self.status = torch.empty(T, 4, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")

    def load(self, i):
        for to, of in zip((self.x, self.gate, self.token), self.inputs[i]):
            to.copy_(of)

    def calls(self):
        """The four calls on torch's current stream."""
        E, s = self.E, self.E.current_stream()
        heads = self.x.view(self.T, self.K // 64, 64)
        self.status.zero_()
        E.ead_qk_norm_rope(self.rope, self.place, heads, None, heads, None, stream=s)
        E.ead_quantise(self.x, self.q, gate=self.gate, stream=s)
        E.ead_linear(self.q, self.w, self.logits, status=self.status, stream=s)
        E.ead_token_logprobs(self.logits, self.token, logprob=self.lp, rank=self.rank, top=self.top, workspace=self.space, status=self.status, stream=s)

    def results(self):
        return [t.clone() for t in (self.x, self.logits, self.lp, self.rank, self.top, self.status)]

    def expected(self):
        """One at a time, with a wait behind each input."""
        out = []
        for i in range(len(self.inputs)):
            self.load(i)
            torch.cuda.synchronize()
            self.calls()
            torch.cuda.synchronize()
            out.append(self.results())
            assert self.status.item() == 0
        return out


def _same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("T", [1, 40, 300])
def test_chain_captured_with_copies_between(E, T):
    """Copies and a memset stand before kernels that start early, in the graph too."""
    c = Chain(E, T, 640, 3000, T)
    want = c.expected()
    stage = [torch.empty_like(t) for t in c.inputs[0]]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        for to, of in zip((c.x, c.gate, c.token), stage):
            to.copy_(of)
        c.calls()
    for i in (0, 1, 2, 3, 1):
        for to, of in zip(stage, c.inputs[i]):
            to.copy_(of)
        g.replay()
        torch.cuda.synchronize()
        assert _same(c.results(), want[i])
    for i in (2, 0, 3):                                                  # replays back to back
        for to, of in zip(stage, c.inputs[i]):
            to.copy_(of)
        g.replay()
        g.replay()
        assert _same(c.results(), want[i])


def test_branches_of_a_graph(E):
    """Two chains side by side in one graph, forked behind one kernel and joined before another."""
    a, b = Chain(E, 70, 640, 5000, 1), Chain(E, 290, 512, 2000, 2)
    want_a, want_b = a.expected(), b.expected()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    total = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        total.add_(1)
        other.wait_stream(side)
        a.calls()
        with torch.cuda.stream(other):
            b.calls()
        side.wait_stream(other)
        a.E.ead_linear(a.q, a.w, a.logits, status=a.status, stream=a.E.current_stream())     # behind both branches
        total.add_(1)
    for i in range(4):
        a.load(i)
        b.load(i)
        g.replay()
        torch.cuda.synchronize()
        assert _same(a.results(), want_a[i]) and _same(b.results(), want_b[i])
    assert total.item() == 8


def test_two_streams_at_once(E):
    chains = [Chain(E, 70, 640, 5000, 1), Chain(E, 290, 512, 2000, 2)]
    want = [c.expected() for c in chains]
    streams = [torch.cuda.Stream() for _ in chains]
    torch.cuda.synchronize()
    got = [[], []]
    for i in (0, 1, 2, 3) * 5:
        for c, s, out in zip(chains, streams, got):
            with torch.cuda.stream(s):
                c.load(i)
                c.calls()
                out.append(c.results())
    torch.cuda.synchronize()
    for out, w in zip(got, want):
        assert all(_same(o, w[i % 4]) for i, o in enumerate(out))


def test_nothing_to_do(E):
    """No rows, no tokens: nothing is launched, nothing is asked of the addresses."""
    empty = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")     # noqa: E731
    none, w = _matrix(E, 0, 256, (1, 128)), _matrix(E, 300, 256, (128, 128))
    E.ead_quantise(empty(0, 256), none, gate=empty(0, 256))
    E.ead_linear(none, w, empty(0, 300))
    E.ead_linear(_matrix(E, 3, 256, (1, 128)), _matrix(E, 0, 256, (128, 128)), empty(3, 0))
    rope = E.ead_rope(torch.zeros(32, device="cuda"), 64)
    E.ead_qk_norm_rope(rope, empty(0, dtype=torch.int32), empty(0, 4, 64), empty(0, 2, 64), empty(0, 4, 64), empty(0, 2, 64))
    E.ead_qk_norm_rope(rope, torch.zeros(3, dtype=torch.int32, device="cuda"), None, None, None, None)
    space = torch.zeros(E.EAD_LOGPROB_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    E.ead_token_logprobs(empty(0, 100), empty(0, dtype=torch.int32), logprob=empty(0, dtype=torch.float32), top=empty(0, 5, dtype=torch.int32), workspace=space)
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim,rot,interleaved", [(128, 128, False), (64, 32, True)])
def test_rotating_write_without_queries(E, fmt, dim, rot, interleaved):
    """The cache gets the same keys and values as beside queries."""
    new, length, heads = [5, 30], [20, 30], 3
    g = torch.Generator().manual_seed(dim)
    n = sum(new)
    both = torch.randn(n, 4 + 2 * heads, dim, generator=g).bfloat16().cuda()
    rope = E.ead_rope(torch.linspace(1, 0.01, rot // 2).cuda(), dim, interleaved=interleaved)
    caches = []
    for q, out in ((both[:, :4], torch.empty(n, 4, dim, dtype=torch.bfloat16, device="cuda")), (None, None)):
        ctx, st = Context(new, length, heads, dim, 16, fmt, seed=1), torch.zeros(1, dtype=torch.int32, device="cuda")
        E.ead_kv_rotate_write(rope, ctx.cache(E), ctx.batch(E), q, both[:, 4:4 + heads], both[:, 4 + heads:], out, status=st)
        assert st.item() == 0
        caches.append(ctx.dev)
    assert all(torch.equal(caches[0][k].view(torch.uint8), caches[1][k].view(torch.uint8)) for k in caches[0])
