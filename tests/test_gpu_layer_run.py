"""The operators of a layer together, as a model runs them: norm, product, head norms, rotated write, attention,
gate, products, logits, draw.  Each stage's outputs are held to its definition on the inputs that it had, which are
the stages' before it; tolerances are those of the stages' own tests.  Then the same captured into graphs, on
other streams, and two at once.
"""
import numpy as np
import pytest
import torch

import test_gpu_linear as linear
import test_gpu_packed as packed
import test_gpu_rotary as rotary
import test_gpu_rows as rows
from oracle import layer
from paper_2608_08020_amd import gambit as g

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 128
E4M3, BF16, F32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32


def _np(t):
    return t.double().cpu().numpy()


class Layer:
    """A layer's weights, with a head of `vocab` tokens."""

    def __init__(self, dim, hq, hkv, hidden, vocab, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)

        def matrix(n, k):
            codes = (64 * torch.randn(n, k, generator=gen, device=DEV)).clamp(-448, 448).to(E4M3)
            scale = (torch.rand(-(-n // 128), -(-k // 128), generator=gen, device=DEV) + 0.5) / 64 / k ** 0.5
            return codes, scale

        def norm(n):
            return (1 + 0.1 * torch.randn(n, generator=gen, device=DEV)).to(BF16)

        self.dim, self.hq, self.hkv, self.hidden = dim, hq, hkv, hidden
        self.qkv, self.o = matrix((hq + 2 * hkv) * D, dim), matrix(dim, hq * D)
        self.up, self.down, self.head = matrix(2 * hidden, dim), matrix(dim, hidden), matrix(vocab, dim)
        self.norms = [norm(dim) for _ in range(3)]
        self.q_norm, self.k_norm = norm(D), norm(D)
        self.table = rotary._table(200, D)

    def heads(self, x, res):
        """Normed, not yet turned queries and keys, and values, of hidden rows x; res takes the sum."""
        codes, scale = g.rms_norm(x, self.norms[0], residual=res, out_dtype=E4M3)
        qkv = g.linear_fp8(codes, scale, *self.qkv)
        q, k, v = qkv.view(-1, self.hq + 2 * self.hkv, D).split([self.hq, self.hkv, self.hkv], 1)
        return (codes, scale), qkv, g.rms_norm(q, self.q_norm), g.rms_norm(k, self.k_norm), v

    def rest(self, att, res):
        """From the attention's output to the normed rows that the head multiplies."""
        s = {"att": att}
        s["a"] = g.quantize(att.reshape(-1, self.hq * D))
        s["o"] = g.linear_fp8(*s["a"], *self.o)
        s["n"] = g.rms_norm(s["o"], self.norms[1], residual=res, out_dtype=E4M3)
        s["up"] = g.linear_fp8(*s["n"], *self.up)
        s["g"] = g.quantize(s["up"], gated=True)
        s["down"] = g.linear_fp8(*s["g"], *self.down)
        s["last"] = g.rms_norm(s["down"], self.norms[2], residual=res, out_dtype=E4M3)
        return s


def _normed(x, w, res):
    return layer.rms_norm(_np(x), _np(w), 1e-6, None if res is None else _np(res))


def _check_rest(m, s, res):
    rows._check_codes(*s["a"], _np(s["att"]).reshape(len(res), -1), 0.0)
    linear._check(s["o"], *s["a"], *m.o)
    # the residual that a norm read is not there any more: it is that before the layer's rest, and the rounded sum
    y, h = _normed(s["o"], m.norms[1], res)
    rows._check_codes(*s["n"], y, rows.REL)
    linear._check(s["up"], *s["n"], *m.up)
    rows._check_codes(*s["g"], layer.gated(_np(s["up"])), 2.0 ** -17)
    linear._check(s["down"], *s["g"], *m.down)
    y, _ = _normed(s["down"], m.norms[2], torch.from_numpy(h).to(F32))
    rows._check_codes(*s["last"], y, rows.REL)


@pytest.mark.parametrize("fp8", [False, True])
def test_prompts_then_single_tokens(fp8):
    hq, hkv, dim = 8, 2, 1024
    m = Layer(dim, hq, hkv, 1280, 5003)
    counts, ids = [1, 23, 40], [0, 1, 2]
    s = packed.Kept(hq, hkv, T=3, maxb=8, fp8=fp8, seed=4)
    s.pool.kv_alloc(ids, counts)
    N = sum(counts)
    x, res = s.normal(N, dim), s.normal(N, dim).float()
    before = res.clone()
    (codes, scale), qkv, q, k, v = m.heads(x, res)
    y, h = _normed(x, m.norms[0], before)
    rows._check_codes(codes, scale, y, rows.REL)
    assert np.abs(_np(res) - h).max() <= 2.0 ** -24 * np.abs(h).max()
    linear._check(qkv, codes, scale, *m.qkv)
    raw = qkv.view(N, hq + 2 * hkv, D)
    rows._check(q, _normed(raw[:, :hq], m.q_norm, None)[0])
    rows._check(k, _normed(raw[:, hq:hq + hkv], m.k_norm, None)[0])
    pos = np.concatenate([np.arange(c) for c in counts])
    turned = s.pool.kv_write_rotated(0, ids, [0] * 3, counts, k, v, m.table, q=q)
    rotary._check(turned, rotary._turned(q, pos, m.table, False))
    kt = rotary._turned(k, pos, m.table, False)
    att = s.pool.prompt_attn(0, ids, counts, turned, out_dtype=BF16)
    base = 0
    for i, c in zip(ids, counts):
        K, V = s.tokens(i, 0, 0, c)
        if not fp8:
            rotary._check(K, (kt[0][base:base + c], kt[1][base:base + c]))
            assert torch.equal(V, v[base:base + c].double())
        packed._check(att[base:base + c], turned[base:base + c], K, V, packed._causal(c, c))
        base += c
    kept = res.clone()
    r = m.rest(att, res)
    _check_rest(m, r, kept)
    # logits of the prompts' last tokens, and the next ones
    at = torch.tensor(np.cumsum(counts) - 1, device=DEV)
    z = g.linear_fp8(r["last"][0][at], r["last"][1][:, at].contiguous(), *m.head, out_dtype=F32)
    linear._check(z, r["last"][0][at], r["last"][1][:, at], *m.head)
    u = torch.tensor([0.1, 0.5, 0.93], device=DEV)
    got = g.sample(z, u, temperature=0.8, top_k=50, top_p=0.95)
    want = [layer.draw(_np(z[j]), float(u[j]), temperature=float(np.float32(0.8)), top_k=50, top_p=float(np.float32(0.95))) for j in range(3)]
    assert got.tolist() == want
    # one token a trace: the one-step attention with turned keys of its own
    held = [s.tokens(i, 0, 0, c) for i, c in zip(ids, counts)]
    x, res = s.normal(3, dim), s.normal(3, dim).float()
    _, _, q, k, v = m.heads(x, res)
    p = torch.tensor(counts, dtype=torch.int32, device=DEV)
    qt, kt = g.rotate(q, k, p, m.table)
    rotary._check(qt, rotary._turned(q, counts, m.table, False))
    rotary._check(kt, rotary._turned(k, counts, m.table, False))
    vd = v.contiguous()
    if not fp8:  # (else the new token is read as its codes stand for it)
        out = s.pool.decode_attn_layer(0, ids, qt, kt, vd, out_dtype=BF16)
        for j, c in enumerate(counts):
            K, V = torch.cat([held[j][0], kt[j:j + 1].double()]), torch.cat([held[j][1], vd[j:j + 1].double()])
            packed._check(out[j:j + 1], qt[j:j + 1], K, V, packed._causal(c + 1, 1))
    else:
        s.pool.kv_alloc(ids, [1] * 3)
        turned = s.pool.kv_write_rotated(0, ids, counts, [1] * 3, k, v, m.table, q=q)
        assert torch.equal(turned, qt)
        out = s.pool.prompt_attn(0, ids, [1] * 3, turned, out_dtype=BF16)
        for j, c in enumerate(counts):
            K, V = s.tokens(ids[j], 0, 0, c + 1)
            assert torch.equal(K[:c], held[j][0])
            packed._check(out[j:j + 1], turned[j:j + 1], K, V, packed._causal(c + 1, 1))
    kept = res.clone()
    _check_rest(m, m.rest(out, res), kept)


def _chain(m, x, res, pos, att, u):
    """The operators that keep nothing, one after another, with new outputs."""
    r = res.clone()
    _, _, q, k, v = m.heads(x, r)
    q, k = g.rotate(q, k, pos, m.table)
    s = m.rest(att, r)
    z = g.linear_fp8(*s["last"], *m.head, out_dtype=F32)
    return q, k, r, z, g.sample(z, u, temperature=0.9, top_k=40), g.sample(z, u, top_p=0.9), g.sample(s["up"], u, min_p=0.01)


def _chain_inputs(m, n, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return [torch.randn(n, m.dim, generator=gen, device=DEV).to(BF16), torch.randn(n, m.dim, generator=gen, device=DEV),
            torch.randint(0, 200, (n,), generator=gen, device=DEV, dtype=torch.int32),
            torch.randn(n, m.hq, D, generator=gen, device=DEV).to(BF16), torch.rand(n, generator=gen, device=DEV)]


@pytest.mark.parametrize("n,vocab", [(3, 5003), (20, 50257), (150, 17000)])
def test_captured_and_replayed_with_other_inputs(n, vocab):
    m = Layer(1024, 8, 2, 1280, vocab)
    args = _chain_inputs(m, n, 0)
    _chain(m, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _chain(m, *args)
    for seed in (1, 2, 1):
        new = _chain_inputs(m, n, seed)
        for a, b in zip(args, new):
            a.copy_(b)
        eager = _chain(m, *new)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)
        _chain(m, *_chain_inputs(m, n, 9))


def test_two_graphs_and_two_streams_at_once():
    m = Layer(1024, 8, 2, 1280, 50257)
    sets = [_chain_inputs(m, n, n) for n in (5, 33)]
    want = [_chain(m, *a) for a in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    graphs, outs = [], []
    for a in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(_chain(m, *a))
    for _ in range(3):
        for s, gr in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
        torch.cuda.synchronize()
        for got, ref in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(got, ref))
    got = []
    for s, a in zip(streams, sets):
        with torch.cuda.stream(s):
            got.append(_chain(m, *a))
    torch.cuda.synchronize()
    for o, ref in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(o, ref))


def test_a_stream_by_argument():
    m = Layer(1024, 8, 2, 1280, 50257)
    x, res, pos, att, u = _chain_inputs(m, 7, 3)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    codes, scale = torch.empty(7, 1024, dtype=E4M3, device=DEV), torch.empty(8, 7, device=DEV)
    z, ids = torch.empty(7, 50257, device=DEV), torch.empty(7, dtype=torch.int32, device=DEV)
    qt = torch.empty(7, 8, D, dtype=BF16, device=DEV)
    torch.cuda.synchronize()
    g.rms_norm(x, m.norms[0], out=codes, out_scale=scale, stream=s)
    g.linear_fp8(codes, scale, *m.head, out=z, stream=s)
    g.sample(z, u, top_p=0.9, out=ids, stream=s)
    g.rotate(att, None, pos, m.table, q_out=qt, stream=s)
    other = [torch.empty(1 << 22, dtype=torch.uint8, device=DEV).fill_(0xA5) for _ in range(8)]  # (not the workspace of the draw)
    torch.cuda.synchronize()
    c2, s2 = g.rms_norm(x, m.norms[0], out_dtype=E4M3)
    z2 = g.linear_fp8(c2, s2, *m.head, out_dtype=F32)
    assert torch.equal(codes.view(torch.uint8), c2.view(torch.uint8)) and torch.equal(scale, s2) and torch.equal(z, z2)
    assert torch.equal(ids, g.sample(z2, u, top_p=0.9)) and torch.equal(qt, g.rotate(att, None, pos, m.table)[0])
    assert len(other) == 8
