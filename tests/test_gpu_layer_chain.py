"""The layer operators as a worker's step uses them: one after another, with the statistics behind them, in graphs, on other
streams, and on matrices whose offsets pass 32 bits.  Tolerances: those of test_gpu_layer_ops.py through the chain, or exact
where every number is a small whole one."""
import numpy as np
import pytest
import torch

import paper_2508_18182_amd as A
from oracle import adloco_oracle as orc
from oracle import layer_oracle as lo
from gpu_util import new_acc, read_acc

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0**-24


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def host(t):
    return t.detach().cpu().double().numpy()


def rand(seed, shape, dtype=torch.bfloat16, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


def values(b):
    return lo.unpack(b.data.cpu().numpy(), b.exponent[:, :b.rows].cpu().numpy(), b.cols)


# ---- per-sample sums as a block of the statistics ---------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,d", [(1, 1), (3, 7), (5, 256), (4, 1000)])
def test_sample_sums_block(ctx, B, d, dtype):
    dt, code = {"f32": (torch.float32, A.ADLOCO_F32), "bf16": (torch.bfloat16, A.ADLOCO_BF16)}[dtype]
    T, wide = 16, 64
    a, delta = rand(1, (B, T, wide), dt), rand(2, (B, T, 32), dt)
    buf = rand(3, (B, d + 3), torch.float32)
    for sums in (buf[:, :d].contiguous(), buf[:, :d], buf[:, 3:]):      # (strided, and not 16-byte aligned)
        v = host(sums)
        g_lin, g_vec = torch.full((32, wide), 9.0, device=DEV), torch.full((d,), 9.0, device=DEV)
        layers = [dict(a=a, delta=delta, grad_sum=g_lin), dict(kind="sample_sums", sums=sums, grad_sum=g_vec)]
        ps, pl, acc = torch.empty(B, device=DEV), torch.empty(2, B, device=DEV), new_acc()
        A.adloco_grad_stats(ctx, layers, B, T, code, ps, pl, acc)
        want = orc.grad_stats([(host(a), host(delta))], two_pass=False)
        norms = (v * v).sum(1)
        np.testing.assert_allclose(host(pl)[1], norms, rtol=1e-6)
        np.testing.assert_allclose(host(ps), want["n_sample"] + norms, rtol=2e-3 if dtype == "bf16" else 1e-4)
        np.testing.assert_allclose(host(g_vec), v.sum(0), rtol=0, atol=1e-6 * np.abs(v).sum(0).max())
        S1, n = read_acc(acc)
        assert n == B and abs(S1 - host(ps).sum()) <= 1e-6 * S1
        res = A.adloco_norm_test(ctx, layers, acc, 0.3, B, 32)
        S2 = (host(g_lin)**2).sum() + (host(g_vec)**2).sum()
        assert abs(res["S2"] - S2) <= 1e-6 * S2
        # a second micro-batch is added, a batch without statistics too
        A.adloco_grad_stats(ctx, layers, B, T, code, ps, pl, acc, A.ADLOCO_ACCUMULATE)
        A.adloco_grad_stats(ctx, layers, B, T, code, None, None, None, A.ADLOCO_ACCUMULATE | A.ADLOCO_SUM_ONLY)
        assert read_acc(acc)[1] == 2 * B
        np.testing.assert_allclose(host(g_vec), 3 * v.sum(0), rtol=0, atol=4e-6 * np.abs(v).sum(0).max())
        # inner products with the batch gradient
        ip, sq, ip_acc = torch.empty(B, device=DEV), torch.empty(B, device=DEV), torch.zeros(4, dtype=torch.float64, device=DEV)
        A.adloco_inner_products(ctx, [layers[1]], B, T, code, ip, sq, ip_acc)
        c = v @ host(g_vec)
        np.testing.assert_allclose(host(ip), c, rtol=0, atol=1e-5 * (np.abs(v) @ np.abs(host(g_vec))).max())
        np.testing.assert_allclose(host(sq), norms, rtol=1e-6)


def test_sample_sums_block_beside_vectors_is_the_vector_block(ctx):
    """Whole numbers: a bias block and the block of its sums over the tokens give the same bits."""
    B, T, d = 6, 20, 300
    delta = torch.randint(-4, 5, (B, T, d)).float().to(DEV)
    got = []
    for block in (dict(kind="vector", delta=delta), dict(kind="sample_sums", sums=delta.sum(1))):
        blocks = [dict(kind="vector", delta=delta, grad_sum=torch.zeros(d, device=DEV)), dict(block, grad_sum=torch.zeros(d, device=DEV)),
                  dict(kind="vector", x=delta, delta=delta, grad_sum=torch.zeros(d, device=DEV))]
        ps, pl, acc = torch.empty(B, device=DEV), torch.empty(3, B, device=DEV), new_acc()
        A.adloco_grad_stats(ctx, blocks, B, T, A.ADLOCO_F32, ps, pl, acc)
        got.append([ps, pl, acc] + [b["grad_sum"] for b in blocks])
    for x, y in zip(*got):
        assert torch.equal(x, y)


def test_sample_sums_refusals(ctx):
    B, T, d = 2, 4, 8
    sums, g = torch.zeros(B, d, device=DEV), torch.zeros(d, device=DEV)
    ps, acc = torch.zeros(B, device=DEV), new_acc()

    def call(**change):
        desc = A.make_layer_descs([dict(kind="sample_sums", sums=sums, grad_sum=g)], B, T, A.ADLOCO_BF16)
        for k, v in change.items():
            setattr(desc[0], k, v)
        A.adloco_grad_stats(ctx, None, B, T, A.ADLOCO_BF16, ps, None, acc, 0, descs=desc)

    call()
    for change in (dict(a=sums.data_ptr()), dict(d_in=2), dict(delta=sums.data_ptr() + 2), dict(delta_row_stride=7), dict(delta=None)):
        with pytest.raises(A.AdlocoError) as e:
            call(**change)
        assert e.value.code == 1
    with pytest.raises(ValueError, match="sums"):
        A.make_layer_descs([dict(kind="sample_sums", sums=sums.bfloat16(), grad_sum=g)], B, T, A.ADLOCO_BF16)


def test_expanded_sample_sums_are_refused(ctx):
    one, g = torch.zeros(8, device=DEV), torch.zeros(8, device=DEV)
    for sums in (one.expand(4, 8), torch.zeros(32, device=DEV).as_strided((4, 8), (4, 1))):
        with pytest.raises(ValueError, match="share memory"):
            A.make_layer_descs([dict(kind="sample_sums", sums=sums, grad_sum=g)], 4, 3, A.ADLOCO_BF16)


def test_round_takes_sample_sums(ctx):
    """adloco_round with a block given by its per-sample sums: the same bits as with the tokens' gradients (whole numbers)."""
    T, d, N = 5, 40, 40 + 8 * 16
    got = []
    for kind in ("vector", "sample_sums"):
        rng = np.random.default_rng(0)
        mk = lambda: torch.from_numpy(rng.normal(size=N).astype(np.float32)).to(DEV)  # noqa: E731
        theta = mk()
        trainer = dict(theta_outer=theta, momentum=torch.zeros(N, device=DEV), b_req=3, acc=new_acc(), uid=0,
                       per_sample_sqnorm=torch.zeros(8, device=DEV),
                       workers=[dict(theta=torch.zeros(N, device=DEV), exp_avg=torch.zeros(N, device=DEV),
                                     exp_avg_sq=torch.zeros(N, device=DEV), grad=torch.zeros(N, device=DEV), step=0) for _ in range(2)])

        def batch(uid, worker, inner, micro, b, theta_ptr):
            r = np.random.default_rng(100 * worker + 10 * inner + micro)
            t = lambda *s: torch.from_numpy(r.integers(-3, 4, s).astype(np.float32)).to(DEV)  # noqa: E731
            delta = t(b, T, d)
            torch.cuda.synchronize()
            first = dict(delta=delta) if kind == "vector" else dict(sums=delta.sum(1))
            return [first, dict(a=t(b, T, 16), delta=t(b, T, 8))]

        cfg = dict(T=T, dtype=A.ADLOCO_F32, inner_steps=2, n_switch=2, merge_w=0, nesterov=1, b_max=8, b_cap=64, eta=0.3,
                   lr_inner=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, lr_outer=0.7, mu_outer=0.9)
        rep = A.adloco_round(ctx, cfg, [trainer], [dict(kind=kind, d_out=d), dict(d_in=16, d_out=8)], batch)
        torch.cuda.synchronize()
        got.append((rep, [theta, trainer["momentum"]] + [w["grad"] for w in trainer["workers"]]))
    assert got[0][0] == got[1][0]
    for x, y in zip(got[0][1], got[1][1]):
        assert torch.equal(x, y)


# ---- one sublayer's step ----------------------------------------------------------------------

class Step:
    """A norm with dropout in front of it and a linear layer behind it, both passes in 8-bit products, and the statistics."""

    def __init__(self, B=3, T=50, d=192, d_out=136, seed=0):
        self.B, self.T, self.d, self.d_out, self.p, self.key = B, T, d, d_out, 0.2, 77
        self.x, self.res = rand(seed + 1, (B, T, d)), rand(seed + 2, (B, T, d), std=2.0)
        self.dy, self.dh_in = rand(seed + 3, (B, T, d_out), std=0.1), rand(seed + 4, (B, T, d), std=0.1)
        self.w = rand(seed + 5, (d_out, d), torch.float32, 0.05)
        self.gain = 1 + 0.1 * rand(seed + 6, (d,), torch.float32)
        new = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device=DEV)  # noqa: E731
        self.h, self.y, self.dn, self.dh, self.dx = (new(B, T, d) for _ in range(5))
        self.out = new(B, T, d_out)
        rows = B * T
        self.y8, self.yt8 = A.Blocks8.empty(rows, d, DEV), A.Blocks8.empty(d, rows, DEV)
        self.w8, self.wt8 = A.Blocks8.empty(d_out, d, DEV), A.Blocks8.empty(d, d_out, DEV)
        self.d8, self.dt8 = A.Blocks8.empty(rows, d_out, DEV), A.Blocks8.empty(d_out, rows, DEV)
        self.g_w, self.g_gain = new(d_out, d, dt=torch.float32), new(d, dt=torch.float32)
        self.sums = new(B, d, dt=torch.float32)
        self.ps, self.acc = new(B, dt=torch.float32), new_acc()
        self.layers = [dict(a=self.y, delta=self.dy, grad_sum=self.g_w, provided=True),
                       dict(kind="sample_sums", sums=self.sums, grad_sum=self.g_gain)]

    def outputs(self):
        return [self.h, self.y, self.out, self.dn, self.dh, self.dx, self.g_w, self.g_gain, self.sums, self.ps, self.acc]

    def clear(self):
        for t in self.outputs():
            t.fill_(3)

    def run(self, ctx, stream=None):
        s = dict(stream=stream)
        A.adloco_pack_blocks(ctx, self.w, self.w8, self.wt8, **s)
        A.adloco_rms_norm(ctx, self.x, self.gain, 1e-5, y=self.y, y8=self.y8, residual=self.res, h_out=self.h, p=self.p, seed=self.key, **s)
        A.adloco_block_product(ctx, self.y8, self.w8, self.out, **s)
        A.adloco_pack_blocks(ctx, self.dy, self.d8, self.dt8, **s)
        A.adloco_pack_blocks(ctx, self.y, None, self.yt8, **s)
        A.adloco_block_product(ctx, self.d8, self.wt8, self.dn, **s)
        A.adloco_block_product(ctx, self.dt8, self.yt8, self.g_w, **s)
        A.adloco_rms_norm_backward(ctx, self.h, self.gain, self.dn, 1e-5, self.dh, gain_sums=self.sums, dh_in=self.dh_in, dx_out=self.dx,
                                   p=self.p, seed=self.key, **s)
        A.adloco_grad_stats(ctx, self.layers, self.B, self.T, A.ADLOCO_BF16, self.ps, None, self.acc, 0, **s)


def test_a_sublayers_step(ctx):
    s = Step()
    s.clear()
    s.run(ctx)
    rows = s.B * s.T
    flat = lambda t: host(t).reshape(rows, -1)  # noqa: E731
    # forward, from the inputs: blocks are 2^-4 off at most, their product by the 2-norm of that over the terms
    h = flat(s.res) + lo.dropout(flat(s.x), s.p, s.key)
    y = lo.rms_norm(h, host(s.gain), 1e-5)
    np.testing.assert_allclose(flat(s.h), h, rtol=2.0**-8, atol=1e-6)
    np.testing.assert_allclose(flat(s.y), y, rtol=2.0**-8, atol=1e-6)
    exact = y @ host(s.w).T
    bound = 2.0**-4 * np.sqrt(2) * np.sqrt((y * y) @ (host(s.w).T**2))      # independent errors of both factors' roundings
    assert np.linalg.norm(flat(s.out) - exact) <= np.linalg.norm(bound) + 2.0**-8 * np.linalg.norm(exact)
    # each later call from what the one before it gave
    near = lambda got, want, cut: np.linalg.norm(got - want) <= cut * np.linalg.norm(want)  # noqa: E731
    assert near(flat(s.out), values(s.y8) @ values(s.w8).T, 2.0**-8)
    assert near(flat(s.dn), values(s.d8) @ values(s.wt8).T, 2.0**-8)
    assert near(host(s.g_w), values(s.dt8) @ values(s.yt8).T, 2e-6)
    grad, parts = lo.rms_norm_backward(flat(s.h), host(s.gain), flat(s.dn), 1e-5)
    dh = grad + flat(s.dh_in)
    assert near(flat(s.dh), dh, 2.0**-8) and near(flat(s.dx), lo.dropout(dh, s.p, s.key), 2.0**-8)
    sums = parts.reshape(s.B, s.T, -1).sum(1)
    np.testing.assert_allclose(host(s.sums), sums, rtol=0, atol=(s.T + 80) * U * np.abs(parts).reshape(s.B, s.T, -1).sum(1).max())
    want = orc.grad_stats([(host(s.y), host(s.dy))], two_pass=False)
    np.testing.assert_allclose(host(s.ps), want["n_sample"] + (host(s.sums)**2).sum(1), rtol=2e-3)
    np.testing.assert_allclose(host(s.g_gain), host(s.sums).sum(0), rtol=0, atol=1e-5 * np.abs(host(s.sums)).sum(0).max())
    # the gradient in 8 bits points where the exact one does
    g = np.einsum("to,td->od", flat(s.dy), y)
    cos = (g * host(s.g_w)).sum() / np.linalg.norm(g) / np.linalg.norm(host(s.g_w))
    assert cos > 1 - 2.0**-7                            # 1 - (2^-4)^2 and the 16-bit roundings


def test_step_in_a_graph_and_on_other_streams():
    ctx = A.Context(0)
    s = Step(seed=20)
    s.clear()
    s.run(ctx)
    torch.cuda.synchronize()
    want = [t.clone() for t in s.outputs()]
    side = torch.cuda.Stream()
    s.clear()
    torch.cuda.synchronize()
    s.run(ctx, stream=side)                             # named stream
    side.synchronize()
    for a, b in zip(s.outputs(), want):
        assert torch.equal(a, b)
    s.clear()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        s.run(ctx)
    for rep in range(4):
        s.clear()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for k, (a, b) in enumerate(zip(s.outputs(), want)):
            assert torch.equal(a, b), (rep, k)
        other = Step(B=2, T=30 + rep, d=264, d_out=72, seed=40 + rep)       # eager work of other shapes in between
        other.run(ctx)
        s.clear()
        s.run(ctx)
        torch.cuda.synchronize()
        for k, (a, b) in enumerate(zip(s.outputs(), want)):
            assert torch.equal(a, b), ("eager", rep, k)
    ctx.close()


def test_without_memory_for_scratch():
    """Sums that would be split are taken whole, eagerly too, and split once there is memory: whole numbers, the same bits."""
    ctx = A.Context(0)
    ctx.set_tuning("scratch_limit_kb", 1)
    a, b = A.Blocks8.empty(64, 20000, DEV), A.Blocks8.empty(72, 20000, DEV)
    x, y = torch.randint(-4, 5, (64, 20000)).float().to(DEV), torch.randint(-4, 5, (72, 20000)).float().to(DEV)
    for m, q in ((x, a), (y, b)):
        A.adloco_pack_blocks(ctx, m, q)
    h, dy = torch.full((500, 64), 2.0, device=DEV), torch.randint(-3, 4, (500, 64)).float().to(DEV)      # h / sqrt(mean(h^2)) = 1
    for limit in (1, 0):
        ctx.set_tuning("scratch_limit_kb", limit)
        out, sums = torch.full((64, 72), 7.0, device=DEV), torch.full((1, 64), 7.0, device=DEV)
        A.adloco_block_product(ctx, a, b, out)
        A.adloco_rms_norm_backward(ctx, h, None, dy, 1e-30, gain_sums=sums)
        np.testing.assert_array_equal(host(out), host(x) @ host(y).T)
        np.testing.assert_allclose(host(sums)[0], host(dy).sum(0), rtol=0, atol=600 * U * 1500)
    ctx.close()


def test_captured_without_scratch_is_right():
    """A context whose first split sum is captured has no scratch for it: it takes the sums whole."""
    ctx = A.Context(0)
    a, b = A.Blocks8.empty(64, 20000, DEV), A.Blocks8.empty(72, 20000, DEV)
    x, y = torch.randint(-4, 5, (64, 20000)).float().to(DEV), torch.randint(-4, 5, (72, 20000)).float().to(DEV)
    for m, q in ((x, a), (y, b)):
        A.adloco_pack_blocks(ctx, m, q)
    out, h, sums = torch.zeros(64, 72, device=DEV), torch.randint(-3, 4, (500, 64)).float().to(DEV), torch.zeros(1, 64, device=DEV)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        A.adloco_block_product(ctx, a, b, out)
        A.adloco_rms_norm_backward(ctx, h, None, h, 1e-5, gain_sums=sums)
    want = host(x) @ host(y).T
    _, parts = lo.rms_norm_backward(host(h), np.ones(64), host(h), 1e-5)
    for rep in range(3):
        out.fill_(7.0)
        sums.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(host(out), want)
        np.testing.assert_allclose(host(sums)[0], parts.sum(0), rtol=0, atol=600 * U * np.abs(parts).sum(0).max())
        # (eager now: scratch is taken, the captured calls keep what they have)
        eager = torch.zeros_like(out)
        A.adloco_block_product(ctx, a, b, eager)
        np.testing.assert_array_equal(host(eager), want)
    ctx.close()


def test_two_contexts_on_two_streams():
    steps, ctxs, streams = [Step(seed=60), Step(seed=70, d=320)], [A.Context(0), A.Context(0)], [torch.cuda.Stream(), torch.cuda.Stream()]
    want = []
    for s, c in zip(steps, ctxs):
        s.run(c)
        torch.cuda.synchronize()
        want.append([t.clone() for t in s.outputs()])
        s.clear()
    torch.cuda.synchronize()
    for _ in range(5):
        for s, c, st in zip(steps, ctxs, streams):
            s.run(c, stream=st)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        for a, b in zip(s.outputs(), w):
            assert torch.equal(a, b)
    for c in ctxs:
        c.close()


def test_micro_batches_keep_their_masks(ctx):
    """SwitchMode may cut a batch: counting first_row on gives every row the mask it has in the whole batch."""
    x, res = rand(5, (96, 200)), rand(6, (96, 200))
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    A.adloco_rms_norm(ctx, x, None, 1e-5, h_out=whole, residual=res, p=0.3, seed=9)
    for a, b in ((0, 40), (40, 41), (41, 96)):
        A.adloco_rms_norm(ctx, x[a:b], None, 1e-5, h_out=parts[a:b], residual=res[a:b], p=0.3, seed=9, first_row=a)
    assert torch.equal(whole, parts)
    alone = torch.empty_like(x)
    A.adloco_dropout(ctx, x, alone, 0.3, 9, residual=res)
    assert torch.equal(whole, alone)
    gone = torch.empty_like(x)                          # every value of a row dropped: h = 0, y = 0
    A.adloco_rms_norm(ctx, x[:, :8], None, 1e-5, y=gone[:, :8], p=65535 / 65536, seed=3)
    keep = torch.from_numpy(lo.dropout_keep(96, 8, 65535 / 65536, 3)).to(DEV)
    assert torch.equal(gone[:, :8] != 0, keep & (x[:, :8] != 0))


# ---- offsets beyond 32 bits -------------------------------------------------------------------

def test_offsets_beyond_32_bits(ctx):
    rows, d = (1 << 21) + 5, 2056                       # 4.3e9 elements, 8.6 GB in bf16
    x = torch.ones(rows, d, dtype=torch.bfloat16, device=DEV)
    last = slice(rows - 3, rows)
    A.adloco_dropout(ctx, x, x, 0.5, 21)
    want = torch.from_numpy(lo.dropout_keep(3, d, 0.5, 21, rows - 3)).to(DEV)
    assert torch.equal(x[last] != 0, want)
    head = torch.from_numpy(lo.dropout_keep(3, d, 0.5, 21)).to(DEV)
    assert torch.equal(x[:3] != 0, head)
    x[last] = rand(7, (3, d))
    ends = x[last].clone()
    small, small8 = torch.empty_like(ends), A.Blocks8.empty(3, d, DEV)
    A.adloco_rms_norm(ctx, ends, None, 1e-5, y=small, y8=small8)
    y8 = A.Blocks8.empty(rows, d, DEV)
    A.adloco_rms_norm(ctx, x, None, 1e-5, y=x, y8=y8)
    assert torch.equal(x[last], small) and torch.equal(y8.data[last], small8.data)
    assert torch.equal(y8.exponent[:, rows - 3:rows], small8.exponent[:, :3])
    w, out, few = A.Blocks8.empty(40, d, DEV), torch.empty(rows, 40, device=DEV), torch.empty(3, 40, device=DEV)
    A.adloco_pack_blocks(ctx, torch.randint(-3, 4, (40, d)).float().to(DEV), w)
    A.adloco_pack_blocks(ctx, x, y8)                    # the norm's own values, packed again
    A.adloco_pack_blocks(ctx, small, small8)
    assert torch.equal(y8.data[last], small8.data)
    A.adloco_block_product(ctx, y8, w, out)
    np.testing.assert_allclose(host(out[last]), values(small8) @ values(w).T, rtol=0, atol=1e-3)
    A.adloco_block_product(ctx, small8, w, few)
    np.testing.assert_allclose(host(few), host(out[last]), rtol=0, atol=1e-3)
    del out
    dh, sums = torch.empty_like(x), torch.empty(1, d, device=DEV)
    A.adloco_rms_norm_backward(ctx, x, None, x, 1e-5, dh, gain_sums=sums)
    grad, _ = lo.rms_norm_backward(host(small), np.ones(d), host(small), 1e-5)
    np.testing.assert_allclose(host(dh[last]), grad, rtol=2.0**-8, atol=2e-6)
