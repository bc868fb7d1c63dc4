"""Tokens one after the other over a paged cache, as they would be generated: a layer's fused
projection, append with rotation, attention, the head's product and the sampled commit.  Every
step is held to float64 on what it read, and captured steps to the eager ones."""

import numpy as np
import pytest
import torch

from paper_2608_26140_amd import acache as A
from tests import paged_reference as R
from tests.test_gpu_paged import check

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
H, G, D, BLOCK, B, VOCAB = 4, 2, 128, 16, 3, 1024
WIDTH = H * D


class Steps:
    """One layer's cache and weights, and the batch's state: the last token of each request, its position, and its
    number of keys once that token is stored."""

    def __init__(self, per=1, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.dims = A.make_dims(WIDTH, H, G, D, 256, "bf16")
        self.per = per
        self.emb = draw(VOCAB, WIDTH).to(BF)
        self.w_qkv, self.w_o, self.w_head = ((draw(n, WIDTH) * WIDTH ** -0.5).to(BF) for n in ((H + 2 * G) * D, WIDTH, VOCAB))
        n_blocks, max_blocks = 40, 8
        self.k, self.v = (torch.full((n_blocks * BLOCK, G * D), float("nan"), dtype=BF, device="cuda") for _ in range(2))
        self.tables = torch.randperm(n_blocks, generator=g, device="cuda")[:B * max_blocks].view(B, max_blocks).to(torch.int32)
        self.cache = A.PagedCache(self.k, self.v, BLOCK, self.tables)
        self.ws = A.paged_workspace(self.dims, self.cache, per)
        n = B * per
        self.ids = torch.randint(VOCAB, (n,), generator=g, device="cuda").to(torch.int32)
        self.u = torch.zeros(n, dtype=torch.float64, device="cuda")
        self.pos = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.key_len = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.conf = torch.zeros(n, device="cuda")
        self.temperature, self.top_p = (torch.full((n,), v, device="cuda") for v in (0.8, 0.95))
        self.top_k = torch.full((n,), 50, dtype=torch.int32, device="cuda")

    def qkv(self, x):
        qkv = A.acache_linear(self.dims, x, self.w_qkv)
        return qkv.split([H * D, G * D, G * D], 1)

    def prompts(self, lens, seed=2):
        """Prompts of unequal length, padded: appended in one call."""
        longest = max(lens)
        x = torch.randn(B * longest, WIDTH, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF)
        at = torch.arange(longest, device="cuda").repeat(B, 1)
        n = torch.tensor(lens, device="cuda")[:, None]
        q, k, v = self.qkv(x)
        A.acache_paged_append(self.dims, self.cache, k, v, torch.where(at < n, at, -1).view(-1).to(torch.int32), longest)
        first = n + torch.arange(self.per, device="cuda")[None, :]
        self.pos.copy_(first.view(-1))
        self.key_len.copy_((first + 1).view(-1))  # a row sees what lies before it, and itself

    def step(self):
        """The rows' next tokens, in place; what the step read and made, for the checks."""
        x = A.acache_gather_rows(self.emb, self.ids)
        q, k, v = self.qkv(x)
        turned = A.acache_paged_append(self.dims, self.cache, k, v, self.pos, self.per, q=q)
        o = A.acache_paged_attention(self.dims, self.cache, turned, self.key_len, self.per, ws=self.ws)
        logits = A.acache_linear(self.dims, A.acache_linear(self.dims, o, self.w_o), self.w_head)
        A.acache_sample_commit(logits, self.u, self.temperature, self.top_k, self.top_p, out=self.ids, conf=self.conf)
        return turned, o, logits

    def advance(self):
        self.pos.add_(self.per)
        self.key_len.add_(self.per)

    def state(self):
        return [t.clone() for t in (self.ids, self.pos, self.key_len, self.k, self.v, self.conf)]

    def restore(self, state):
        for t, s in zip((self.ids, self.pos, self.key_len, self.k, self.v, self.conf), state):
            t.copy_(s)


def u_of(step, n):
    return torch.rand(n, dtype=torch.float64, generator=torch.Generator().manual_seed(100 + step))


@pytest.mark.parametrize("per", [1, 3])
def test_steps_against_float64(per):
    m = Steps(per)
    m.prompts([29, 1, 16])
    for i in range(12):
        u = u_of(i, B * per)
        m.u.copy_(u)
        turned, o, logits = m.step()
        ref = R.attention(turned.cpu(), m.key_len.cpu(), m.k.cpu(), m.v.cpu(), BLOCK, m.tables.cpu(), H, G, D, per)
        check(o, ref[0], ref[2], f"step {i}")
        n = B * per
        want, conf, _ = R.sample(logits.double().cpu().numpy(), u.numpy(), np.full(n, np.float32(0.8)), np.full(n, 50),
                                 np.full(n, np.float32(0.95)), None, m.ids.cpu().numpy())
        assert np.array_equal(m.ids.cpu().numpy(), want)
        assert np.all(np.abs(m.conf.cpu().numpy() - conf) <= 2.0 ** -23 * conf)
        m.advance()
    # what the steps stored is the prompts' and their own rows, nothing else
    stored = torch.zeros(m.k.shape[0], dtype=torch.bool)
    for b, first in enumerate((29, 1, 16)):
        for p in range(first + 12 * per):
            stored[R.slot(m.tables.cpu(), 40, BLOCK, b, p)] = True
    assert torch.equal(torch.isfinite(m.k).all(1).cpu(), stored) and torch.isnan(m.k[~stored.cuda()]).all()


def test_captured_steps_follow_the_eager_ones():
    """Two graphs that share a workspace, replayed in turn among eager work and synchronisations: lengths, positions
    and tokens move on the device."""
    m = Steps()
    m.prompts([40, 7, 100])
    begin = m.state()
    steps = 10

    def eager():
        m.restore(begin)
        tokens = []
        for i in range(steps):
            m.u.copy_(u_of(i, B))
            m.step()
            m.advance()
            tokens.append(m.ids.clone())
        return torch.stack(tokens), m.state()
    want, after = eager()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.step()
            m.advance()
        graphs.append(g)
    for round_ in range(2):
        m.restore(begin)
        for i in range(steps):
            m.u.copy_(u_of(i, B))
            graphs[i % 2].replay()
            assert torch.equal(m.ids, want[i]), f"round {round_} step {i}"
            if i == 4:  # eager work between
                keep, u = m.state(), m.u.clone()
                again, _ = eager()
                assert torch.equal(again, want)
                m.restore(keep)
                m.u.copy_(u)
        torch.cuda.synchronize()
        got = m.state()
        for a, b in zip(got, after):
            assert torch.equal(a.view(torch.uint8 if a.dtype == BF else a.dtype), b.view(torch.uint8 if b.dtype == BF else b.dtype))


def test_results_belong_to_the_stream_of_the_call():
    m = Steps()
    m.prompts([30, 20, 10])
    side = torch.cuda.Stream()
    here = torch.cuda.current_stream().cuda_stream
    x = torch.randn(B, WIDTH, device="cuda").to(BF)
    q, k, v = m.qkv(x)
    big = torch.randn(200, 40000, device="cuda").to(BF)
    u = torch.rand(200, dtype=torch.float64, device="cuda")
    turned = A.acache_paged_append(m.dims, m.cache, k, v, m.pos, 1, q=q)

    def stream_of(t):
        for seg in torch.cuda.memory_snapshot():
            if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
                return seg["stream"]
    for name, call in {
            "append": lambda s: A.acache_paged_append(m.dims, m.cache, k, v, m.pos, 1, q=q, stream=s),
            "attention": lambda s: A.acache_paged_attention(m.dims, m.cache, turned, m.key_len, 1, ws=m.ws, stream=s),
            "sample": lambda s: A.acache_sample_commit(big, u, stream=s)}.items():
        want = call(None)
        torch.cuda.synchronize()
        got = call(side)
        side.synchronize()
        assert torch.equal(got, want), name
        assert stream_of(want) == here and stream_of(got) == side.cuda_stream, name
