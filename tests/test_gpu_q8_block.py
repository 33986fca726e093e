"""The 8-bit operators as a block uses them, one after the other: each against fp64 on what it was really given, the whole captured and
replayed, and the models that run on them."""
import gc

import pytest
import torch

from paper_2603_05959_b200 import binding as B
from paper_2603_05959_b200 import harness as H
from paper_2603_05959_b200 import inputs as gen

pytestmark = pytest.mark.gpu


class Block:
    """Norm, QKV, cache, attention, output product, norm, MLP: `seqs` sequences, M tokens of each a step, in buffers of its own."""

    def __init__(self, seqs, M, heads, capacity, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
        C = heads * 64
        self.shape, self.heads, self.C = (seqs, M), heads, C
        weight = lambda n, k: B.k_norm_q8((rnd(n, k) * 0.05).bfloat16(), kind=B.NORM_NONE)
        self.qkv, self.o, self.fc1, self.fc2 = weight(3 * C, C), weight(C, C), weight(4 * C, C), weight(C, 4 * C)
        self.g1, self.g2 = (1 + 0.1 * rnd(C)).bfloat16(), (1 + 0.1 * rnd(C)).bfloat16()
        self.cache = B.new_cache_q8(seqs, capacity, heads)
        self.lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(16, dtype=torch.int32, device="cuda")
        self.x = torch.zeros((seqs * M, C), dtype=torch.bfloat16, device="cuda")
        self.r = torch.zeros_like(self.x)

    def step(self, live=None):
        """One step from x and the branch r that is still to be added to it; everything it made, by name."""
        (seqs, M), C = self.shape, self.C
        new = lambda width: torch.empty((seqs * M, width), dtype=torch.bfloat16, device="cuda")
        t = dict(h=new(C), q=new(C), k=new(C), v=new(C), up=new(4 * C), mid=new(C), out=new(C))
        t["a"], t["a_scale"] = B.k_norm_q8(self.x, weight=self.g1, residual=self.r, sum_out=t["h"])
        B.k_linear_q8(t["a"], t["a_scale"], *self.qkv, (t["q"], t["k"], t["v"]), status=self.status)
        by_seq = lambda y: y.view(seqs, M, C)
        B.k_store_q8(self.cache, by_seq(t["k"]), by_seq(t["v"]), start=self.lens)
        self.lens += M
        t["att"] = B.k_attention_q8(by_seq(t["q"]), self.cache, lens=self.lens, live=live, status=self.status)
        t["b"], t["b_scale"] = B.k_norm_q8(t["att"].view(seqs * M, C), kind=B.NORM_NONE)
        B.k_linear_q8(t["b"], t["b_scale"], *self.o, (), residual=t["h"], sum_out=t["mid"], status=self.status)
        t["c"], t["c_scale"] = B.k_norm_q8(t["mid"], weight=self.g2, kind=B.NORM_LAYER)
        B.k_linear_q8(t["c"], t["c_scale"], *self.fc1, (t["up"],), gelu=True, status=self.status)
        t["d"], t["d_scale"] = B.k_norm_q8(t["up"], kind=B.NORM_NONE)
        B.k_linear_q8(t["d"], t["d_scale"], *self.fc2, (), residual=t["mid"], sum_out=t["out"], status=self.status)
        return t


def _rows_close(q, scale, y):
    torch.testing.assert_close(scale.double(), y.abs().amax(-1) / 127, rtol=2e-5, atol=0)
    assert float((q.double() - y / scale.double()[:, None]).abs().max()) <= 0.5 + 127 * 3e-5       # (half a step, and the row's own rounding)


def _product(a, a_scale, w):
    return ((a.double() @ w[0].double().T).float() * a_scale[:, None] * w[1]).bfloat16()


@pytest.mark.parametrize("seqs,M,heads,steps", [(3, 1, 4, 5), (2, 40, 6, 2), (1, 333, 4, 2)])
def test_each_step_from_what_it_was_given(seqs, M, heads, steps):
    blk = Block(seqs, M, heads, capacity=(steps * M + 15) // 16 * 16)
    g = torch.Generator(device="cuda").manual_seed(M)
    for n in range(1, steps + 1):
        blk.x.copy_(torch.randn(blk.x.shape, generator=g, device="cuda"))
        blk.r.copy_(torch.randn(blk.x.shape, generator=g, device="cuda"))
        t = blk.step()
        h = blk.x + blk.r
        assert torch.equal(t["h"], h)
        y = h.double()
        _rows_close(t["a"], t["a_scale"], y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * blk.g1.double())
        qkv = _product(t["a"], t["a_scale"], blk.qkv)
        assert torch.equal(torch.cat([t["q"], t["k"], t["v"]], 1), qkv)
        # the rows in the cache are within half a step, 2^-7 of the power of two below a block's largest, of k and v (at the largest one a whole one)
        k, v = B.k_load_q8(blk.cache, n * M, dtype=torch.float32)
        for got, want in ((k, t["k"]), (v, t["v"])):
            new, want = got[:, (n - 1) * M:].reshape(-1, 64).double(), want.double().view(-1, 64)
            assert bool(((new - want).abs() <= 2.0 ** -6 * want.abs().amax(-1, keepdim=True)).all())
        q = t["q"].double().view(seqs, M, heads, 64).transpose(1, 2)
        kd, vd = (x.double().view(seqs, n * M, heads, 64).transpose(1, 2) for x in (k, v))
        p = torch.softmax(q @ kd.transpose(2, 3) / 8, -1)
        ref = (p @ vd).transpose(1, 2).reshape(seqs * M, -1)
        spread = (p @ vd.abs()).transpose(1, 2).reshape(seqs * M, -1)
        # (the tolerance of the attention's own tests: P in bf16, Q as whole numbers, the result's rounding)
        dq = (q.abs().amax(-1, keepdim=True) * kd.abs().sum(-1).amax(-1)[:, :, None, None] * 2.0 ** -14 / 8).expand_as(q).transpose(1, 2).reshape(seqs * M, -1)
        att = t["att"].view(seqs * M, -1)
        assert bool(((att.double() - ref).abs() <= (torch.expm1(2 * dq) + 2.0 ** -8 + 1e-5) * spread + 2.0 ** -8 * ref.abs()).all())
        _rows_close(t["b"], t["b_scale"], att.double())
        assert torch.equal(t["mid"], t["h"] + _product(t["b"], t["b_scale"], blk.o))
        y = t["mid"].double()
        y = y - y.mean(-1, keepdim=True)
        _rows_close(t["c"], t["c_scale"], y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * blk.g2.double())
        up = _product(t["c"], t["c_scale"], blk.fc1).double()
        up = 0.5 * up * torch.special.erfc(-up / 2 ** 0.5)
        assert bool(((t["up"].double() - up).abs() <= (2.0 ** -8 + 1e-5) * up.abs() + 1e-17).all())
        _rows_close(t["d"], t["d_scale"], t["up"].double())
        assert torch.equal(t["out"], t["mid"] + _product(t["d"], t["d_scale"], blk.fc2))
    assert int(blk.status[0]) == 0 and blk.lens.tolist() == [steps * M] * seqs


@pytest.mark.parametrize("seqs,M", [(4, 1), (1, 1100)])
def test_captured_and_replayed(seqs, M):
    """A captured step, replayed on new inputs while the cache grows, gives the bits of the same steps made one by one; a second graph of another
    block, replayed on another stream meanwhile, does not disturb it."""
    steps = 4
    blocks = [Block(seqs, M, 4, capacity=steps * M + 16, seed=s) for s in (0, 0, 1)]
    g = torch.Generator(device="cuda").manual_seed(5)
    xs = torch.randn((steps, *blocks[0].x.shape), generator=g, device="cuda").bfloat16()
    rs = torch.randn((steps, *blocks[0].x.shape), generator=g, device="cuda").bfloat16()
    eager, captured, other = blocks
    want = []
    for i in range(steps):
        eager.x.copy_(xs[i])
        eager.r.copy_(rs[i])
        want.append(eager.step()["out"].clone())
    graphs, outs = [], []
    for blk in (captured, other):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            blk.step()                                     # (what is set up on a first call)
        side.synchronize()
        blk.lens.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(blk.step()["out"])
        graphs.append(graph)
    torch.cuda.synchronize()
    beside = torch.cuda.Stream()
    for i in range(steps):
        captured.x.copy_(xs[i])
        captured.r.copy_(rs[i])
        with torch.cuda.stream(beside):
            graphs[1].replay()
        graphs[0].replay()
        assert torch.equal(outs[0], want[i])
    torch.cuda.synchronize()
    assert int(captured.status[0]) == 0 and captured.lens.tolist() == eager.lens.tolist()


def _frames(cfg, n):
    g = torch.Generator(device="cuda").manual_seed(3)
    M = cfg.tokens_per_frame
    return (torch.randn((n, M, cfg.dim), generator=g, device="cuda").bfloat16(), torch.rand(cfg.grid_h * cfg.grid_w, generator=g, device="cuda"),
            [torch.randn((M, cfg.dim), generator=g, device="cuda").bfloat16() for _ in range(cfg.n_layers)])


@pytest.mark.parametrize("model", [H.ProjectionStack, H.Aggregator], ids=["stack", "aggregator"])
def test_models_in_8_bits(model):
    """A model with its products in 8 bits beside the same one in bf16.  A rounding to 8 bits is off by at most half a step, amax / 254, or
    amax / (254 sqrt(3)) in the mean of its square; over a row of up to 1024 normal values amax is under 5 deviations: 1.2 %, and 1.6 % for a
    product of two.  A branch of a block chains two or three of them, 2.8 %, its attention averages; what it is added to has no error: the sums of two
    branches of a layer stay within 6 %."""
    cfg = gen.StreamConfig(name="8 bits", n_layers=1, n_heads=4, grid_h=9, grid_w=15, budget=400, anchor_tokens=0)
    xs, conf, resid = _frames(cfg, 4)
    got = []
    for kind in ("library", "int8"):
        m = model(cfg, torch.device("cuda"), matmul=kind)
        out = []
        for t in range(4):
            args = (xs[t], conf, 0.9) if model is H.Aggregator else (xs[t], resid, conf, 0.9)
            out.append(m.frame(t, *args, torch.cuda.current_stream()).float())
        got.append(torch.stack(out))
        m.destroy()
        del m
    gc.collect()
    assert float((got[1] - got[0]).norm()) <= 0.06 * float(got[0].norm())
    assert not torch.equal(got[0], got[1])


@pytest.mark.parametrize("model", [H.ProjectionStack, H.Aggregator], ids=["stack", "aggregator"])
def test_hooks_of_models_in_8_bits_keep_what_they_are_given(model):
    cfg = gen.StreamConfig(name="hooks", n_layers=2, n_heads=2, grid_h=9, grid_w=15, budget=400, anchor_tokens=0)
    xs, conf, resid = _frames(cfg, 2)
    m, kept, seen = model(cfg, torch.device("cuda"), matmul="int8"), [], []

    def tap(t, l, *tensors):
        kept.append(tensors)
        seen.append([x.clone() for x in tensors])

    m.tap = tap
    for t in range(2):
        args = (xs[t], conf, 0.9) if model is H.Aggregator else (xs[t], resid, conf, 0.9)
        m.frame(t, *args, torch.cuda.current_stream())
    assert len(kept) == 4 and all(torch.equal(p, q) for a, b in zip(kept, seen) for p, q in zip(a, b))
    m.destroy()
    del m, tap, args
    gc.collect()
