"""The dense operators on the GPU against their plain 64-bit forms: 8-bit rows (codes and scales
equal), 8-bit products, the gated block on 8-bit and on 16-bit weights, and its gradients."""
import pytest
import torch

from tests import dense_common as D
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
# rows, output features, depth: one token to ragged batches, sizes off every tile and alignment
SIZES = [(1, 1, 1), (1, 5, 3), (1, 64, 64), (1, 130, 2048), (2, 64, 130), (3, 129, 77), (5, 48, 1000), (8, 256, 512),
         (12, 100, 264), (16, 33, 1001), (17, 96, 72), (33, 520, 136), (64, 200, 1024), (65, 31, 513), (100, 300, 999),
         (128, 128, 192), (257, 136, 320), (300, 700, 640), (520, 513, 257)]
# several tiles in every direction; more tiles than compute units in h, in the gradients of the weights, in dx
LARGE = [(600, 1088, 768), (1025, 520, 1096), (2100, 264, 512), (4000, 4500, 72), (40, 6000, 1800), (6100, 40, 3400)]


def _guarded(shape, dtype):
    """An output with 64 elements behind it, and the check that they are left alone."""
    n = 1
    for s in shape:
        n *= s
    pad = (16 // dtype.itemsize) - n % (16 // dtype.itemsize)
    buf = torch.full((n + pad + 64,), 77, dtype=dtype, device="cuda")
    return buf[:n].view(shape), lambda: bool((buf[n:] == 77).all())


def _rows8(P, q, s):
    return P.Int8Rows(q.to(torch.int8).cuda(), s.cuda())


def _codes(seed, n, k):
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(-127, 128, (n, k), generator=g)
    return q, torch.rand(n, generator=g) * 0.02 + 1e-3


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("m,k", [(1, 1), (1, 7), (3, 8), (2, 255), (5, 256), (4, 1001), (130, 768), (7, 4099),
                                 (3, 20000), (2, 70001), (1, 28672)])
def test_quantize_rows(dtype, m, k):
    require_gpu()
    import paper_2510_03275_amd as P
    x = (D.rand(m * k, m, k) * torch.exp(D.rand(k, m, 1) * 2)).to(dtype)
    ref_q, ref_s = D.quantize_ref(x)
    q, ok_q = _guarded((m, k), torch.int8)
    s, ok_s = _guarded((m,), F32)
    r = P.int8_quantize(x.cuda(), out=P.Int8Rows(q, s))
    assert torch.equal(r.scales.cpu(), ref_s) and torch.equal(r.q.cpu().long(), ref_q)
    assert ok_q() and ok_s()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_quantize_special_rows(dtype):
    """Halves (ties to even), zeros, the smallest numbers, infinities and NaN, at both ends of a row."""
    require_gpu()
    import paper_2510_03275_amd as P
    k = 530
    x = torch.zeros(12, k, dtype=dtype)
    x[0] = torch.arange(-264, 266).to(dtype) / 2            # halves; the largest is 132.5
    x[1, :254] = torch.arange(-127, 127).to(dtype) + 0.5
    x[1, 300] = 127.0                                        # scale one: every x a tie
    x[2, 7] = torch.finfo(dtype).smallest_normal
    x[3, 529] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    x[4] = torch.finfo(dtype).max
    x[5, 0], x[6, 529], x[7, 100], x[8, 529] = float("inf"), float("-inf"), float("nan"), float("nan")
    x[9] = -torch.finfo(dtype).max
    x[10, 528] = -3.0
    ref_q, ref_s = D.quantize_ref(x)
    r = P.int8_quantize(x.cuda())
    assert torch.equal(r.scales.cpu().view(torch.int32)[:5], ref_s.view(torch.int32)[:5])
    assert torch.equal(torch.isnan(r.scales.cpu()), torch.isnan(ref_s))
    assert torch.equal(torch.nan_to_num(r.scales.cpu()), torch.nan_to_num(ref_s))
    assert torch.equal(r.q.cpu().long(), ref_q)
    w = _rows8(P, *_codes(1, 40, k))
    y = P.int8_linear(x.cuda(), w, dtype=F32)
    for i in range(12):      # one row: quantised by the product itself
        one = P.int8_linear(x[i:i + 1].cuda(), w, dtype=F32)
        assert torch.equal(one.nan_to_num(7), y[i:i + 1].nan_to_num(7)), i
    assert torch.equal(torch.isnan(y).all(1).cpu(), torch.isnan(ref_s))
    assert not bool(torch.isnan(y[:5]).any())


@pytest.mark.parametrize("m,n,k", SIZES + LARGE)
@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, F32), (F32, BF16)])
def test_int8_linear(m, n, k, dtype, out):
    require_gpu()
    import paper_2510_03275_amd as P
    x = D.rand(m + n + k, m, k).to(dtype)
    wq, sw = _codes(k, n, k)
    w = _rows8(P, wq, sw)
    q, s = D.quantize_ref(x)
    ref = D.int8_ref(q, s, wq, sw)
    bound = (D.half(out) + 2.0 ** -22) * ref.abs() + D.floor(out)   # fp32: the sum and two products rounded
    y, ok = _guarded((m, n), out)
    P.int8_linear(x.cuda(), w, out=y)
    D.assert_close(y, ref, bound, "quantised by the call")
    y2 = P.int8_linear(P.int8_quantize(x.cuda()), w, dtype=out)
    assert torch.equal(y, y2) and ok()
    base = D.rand(7, m, n).to(out)
    acc, ok = _guarded((m, n), out)
    acc.copy_(base)
    P.int8_linear(x.cuda(), w, out=acc, accumulate=True)
    ref = ref + base.double()
    D.assert_close(acc, ref, bound + (D.half(out) + 2.0 ** -22) * (ref.abs() + base.double().abs()), "accumulated")
    assert ok()


@pytest.mark.parametrize("m", [1, 4, 20, 200])
def test_int8_sums_are_exact(m):
    """The largest sums that 32 bits hold, in every path's order: k = 131071 codes of -128."""
    require_gpu()
    import paper_2510_03275_amd as P
    n, k = 70, D.INT8_MAX_K
    q = torch.full((m, k), -128, dtype=torch.int8)
    q[:, 5] = 1
    w = torch.full((n, k), -128, dtype=torch.int8)
    w[:, 9] = 3
    one = torch.ones(max(m, n))
    y = P.int8_linear(P.Int8Rows(q.cuda(), one[:m].cuda()), P.Int8Rows(w.cuda(), one[:n].cuda()), dtype=F32)
    want = 128 * 128 * (k - 2) - 128 - 3 * 128
    assert bool((y.cpu() == torch.tensor(float(want), dtype=F32)).all())


@pytest.mark.parametrize("m,f,k", SIZES + LARGE)
@pytest.mark.parametrize("dtype,out,act", [(F16, F16, 0), (BF16, BF16, 1), (F32, F32, 0)])
def test_int8_gated_linear(m, f, k, dtype, out, act):
    require_gpu()
    import paper_2510_03275_amd as P
    x = D.rand(m + f + k, m, k).to(dtype)
    (gq, gs), (uq, us) = _codes(k, f, k), _codes(k + 1, f, k)
    gs, us = gs / k ** 0.5, us / k ** 0.5
    q, s = D.quantize_ref(x)
    g, u = D.int8_ref(q, s, gq, gs), D.int8_ref(q, s, uq, us)
    ref, bound = D.gated_bound(g, u, 2.0 ** -22 * g.abs(), 2.0 ** -22 * u.abs(), act, out)
    h, ok = _guarded((m, f), out)
    P.int8_gated_linear(x.cuda(), _rows8(P, gq, gs), _rows8(P, uq, us), act, out=h)
    D.assert_close(h, ref, bound)
    assert ok()


@pytest.mark.parametrize("m,f,k", SIZES + LARGE)
@pytest.mark.parametrize("dtype,act", [(F16, 1), (BF16, 0)])
def test_gated_linear(m, f, k, dtype, act):
    require_gpu()
    import paper_2510_03275_amd as P
    x = D.rand(m + f + k, m, k).to(dtype)
    wg, wu = (D.rand(f, f, k, scale=k ** -0.5).to(dtype), D.rand(f + 1, f, k, scale=k ** -0.5).to(dtype))
    g, u, eg, eu = D.gated_ref(x, wg, wu, act)
    ref, bound = D.gated_bound(g, u, eg, eu, act, dtype)
    h, ok = _guarded((m, f), dtype)
    P.gated_linear(x.cuda(), wg.cuda(), wu.cuda(), act, out=h)
    D.assert_close(h, ref, bound, "h")
    (h2, ok2), (kg, ok3), (ku, ok4) = (_guarded((m, f), dtype) for _ in range(3))
    P.gated_linear(x.cuda(), wg.cuda(), wu.cuda(), act, out=h2, g=kg, u=ku)
    assert torch.equal(h, h2) and ok() and ok2() and ok3() and ok4()
    D.assert_close(kg, g, eg + D.half(dtype) * (g.abs() + eg) + D.floor(dtype), "g")
    D.assert_close(ku, u, eu + D.half(dtype) * (u.abs() + eu) + D.floor(dtype), "u")
    (kg, ok3), (ku, ok4) = (_guarded((m, f), F32) for _ in range(2))
    P.gated_linear(x.cuda(), wg.cuda(), wu.cuda(), act, out=h2, g=kg, u=ku)
    assert torch.equal(h, h2) and ok2() and ok3() and ok4()
    D.assert_close(kg, g, eg, "g in fp32")
    D.assert_close(ku, u, eu, "u in fp32")


@pytest.mark.parametrize("m,f,k", SIZES + LARGE)
@pytest.mark.parametrize("dtype,act", [(F16, 0), (BF16, 1)])
def test_gated_backward(m, f, k, dtype, act):
    require_gpu()
    import paper_2510_03275_amd as P
    x = D.rand(m + f + k, m, k).to(dtype)
    wg, wu = (D.rand(f, f, k, scale=k ** -0.5).to(dtype), D.rand(f + 1, f, k, scale=k ** -0.5).to(dtype))
    g, u, dh = ((D.rand(m + i, m, f) * 2).to(dtype) for i in range(3))
    base = [D.rand(i, f, k).to(dtype) for i in (3, 4)]
    dev = [v.cuda() for v in (dh, x, wg, wu, g, u)]
    outs = [_guarded(s, dtype) for s in ((m, k), (f, k), (f, k))]
    dx, dg, du = (o[0] for o in outs)
    P.gated_linear_backward(*dev, act, dx=dx, dgate=dg, dup=du)
    ref = D.backward_ref(dh, x, wg, wu, g, u, act, dtype)
    for got, (r, b), what in zip((dx, dg, du), ref, ("dx", "dgate", "dup")):
        D.assert_close(got, r, b, what)
    # parts alone are the same bits
    a, b, c = P.gated_linear_backward(*dev, act, need_weights=False)
    assert torch.equal(a, dx) and b is None and c is None
    a, b, c = P.gated_linear_backward(*dev, act, need_dx=False)
    assert a is None and torch.equal(b, dg) and torch.equal(c, du)
    assert all(o[1]() for o in outs)
    g32, u32 = ((D.rand(m + i, m, f) * 2).float() for i in range(1, 3))
    got = P.gated_linear_backward(*dev[:4], g32.cuda(), u32.cuda(), act)
    for v, (r, b), what in zip(got, D.backward_ref(dh, x, wg, wu, g32, u32, act, dtype), ("dx", "dgate", "dup")):
        D.assert_close(v, r, b, what + " from g and u in fp32")
    dg.copy_(base[0])
    du.copy_(base[1])
    P.gated_linear_backward(*dev, act, dgate=dg, dup=du, accumulate=True)
    ref = D.backward_ref(dh, x, wg, wu, g, u, act, dtype, base)
    for got, (r, b), what in zip((dg, du), ref[1:], ("dgate", "dup")):
        D.assert_close(got, r, b, what + " accumulated")
    assert all(o[1]() for o in outs)


@pytest.mark.parametrize("act", [0, 1])
def test_activation_far_out(act):
    """Projections up to the ends of bf16: saturated, no NaN, the gradient 0 or 1 there."""
    require_gpu()
    import paper_2510_03275_amd as P
    vals = torch.tensor([0.0, 1e-30, 1.0, -1.0, 5.0, -5.0, 30.0, -30.0, 90.0, -90.0, 1e4, -1e4, 1e15, -1e15, 1e30, -1e30,
                         3e38, -3e38], dtype=BF16)
    f = vals.numel()
    x = torch.ones(1, 1, dtype=BF16)
    wg = vals[:, None].contiguous()
    wu = torch.full((f, 1), 0.5, dtype=BF16)
    h = P.gated_linear(x.cuda(), wg.cuda(), wu.cuda(), act).cpu().double()
    g = vals.double()[None]
    a, da = D.act_ref(g.clamp(-1e10, 1e10), act)
    a = torch.where(g > 1e9, g, a)
    a = torch.where(g < -1e9, torch.zeros_like(a), a)
    da = torch.where(g.abs() > 1e9, (g > 0).double(), da)
    # e^-a underflows or overflows in fp32 from |a| = 87 on: act(g) is |g| e^-87 at most there
    assert bool(((h - 0.5 * a).abs() <= 2.0 ** -8 * 0.5 * a.abs() + 1e-35).all())
    one = torch.ones(1, f, dtype=BF16)
    dx, dg, du = P.gated_linear_backward(one.cuda(), x.cuda(), wg.cuda(), wu.cuda(), vals[None].cuda(),
                                         (one * 0.5).cuda(), act)
    assert bool(((dg.cpu().double()[:, 0] - 0.5 * da[0]).abs() <= 2.0 ** -8 * 0.5 * da[0].abs() + 2.0 ** -17).all())
    assert bool(((du.cpu().double()[:, 0] - a[0]).abs() <= 2.0 ** -8 * a[0].abs() + 1e-35).all())


@pytest.mark.parametrize("m", [1, 20, 300])
def test_nan_stays_in_its_row(m):
    require_gpu()
    import paper_2510_03275_amd as P
    f, k = 200, 520
    x = D.rand(1, m, k).to(BF16)
    x[0, k - 1] = float("nan")
    wg, wu = (D.rand(i, f, k, scale=0.05).to(BF16) for i in (2, 3))
    h = P.gated_linear(x.cuda(), wg.cuda(), wu.cuda())
    assert bool(torch.isnan(h[0]).all()) and not bool(torch.isnan(h[1:]).any())


def test_empty():
    require_gpu()
    import paper_2510_03275_amd as P
    z = lambda *s: torch.zeros(*s, dtype=F16, device="cuda")
    assert P.int8_quantize(z(0, 5)).q.shape == (0, 5)
    w0 = P.int8_quantize(z(0, 8))
    w = P.int8_quantize(torch.ones(3, 8, device="cuda"))
    assert P.int8_linear(z(0, 8), w).shape == (0, 3) and P.int8_linear(z(2, 8), w0).shape == (2, 0)
    assert P.int8_gated_linear(z(0, 8), w, w).shape == (0, 3) and P.int8_gated_linear(z(2, 8), w0, w0).shape == (2, 0)
    assert P.gated_linear(z(0, 8), z(3, 8), z(3, 8)).shape == (0, 3)
    assert P.gated_linear(z(2, 8), z(0, 8), z(0, 8)).shape == (2, 0)
    out = [torch.full((3, 8), 5.0, dtype=F16, device="cuda") for _ in range(2)]
    P.gated_linear_backward(z(0, 3), z(0, 8), z(3, 8), z(3, 8), z(0, 3), z(0, 3), dgate=out[0], dup=out[1],
                            accumulate=True)
    assert bool((out[0] == 5).all()) and bool((out[1] == 5).all())
    _, dg, du = P.gated_linear_backward(z(0, 3), z(0, 8), z(3, 8), z(3, 8), z(0, 3), z(0, 3), dgate=out[0], dup=out[1])
    assert not bool(dg.any()) and not bool(du.any())
    dx = torch.full((2, 8), 5.0, dtype=F16, device="cuda")
    P.gated_linear_backward(z(2, 0), z(2, 8), z(0, 8), z(0, 8), z(2, 0), z(2, 0), dx=dx)
    assert not bool(dx.any())


@pytest.mark.parametrize("k", [7, 9, 40])
def test_empty_sums(k):
    """No rows: zero gradients of the weights; no features: a zero dx (rows aligned and not)."""
    require_gpu()
    import paper_2510_03275_amd as P
    z = lambda *s: torch.zeros(*s, dtype=BF16, device="cuda")
    out = [torch.full((5, k), 5.0, dtype=BF16, device="cuda") for _ in range(2)]
    P.gated_linear_backward(z(0, 5), z(0, k), z(5, k), z(5, k), z(0, 5), z(0, 5), dgate=out[0], dup=out[1])
    assert not any(bool(o.any()) for o in out)
    dx = torch.full((70, k), 5.0, dtype=BF16, device="cuda")
    P.gated_linear_backward(z(70, 0), z(70, k), z(0, k), z(0, k), z(70, 0), z(70, 0), dx=dx)
    assert not bool(dx.any())


@pytest.mark.parametrize("m,f,k", [(1, 48, 64), (16, 96, 1001), (24, 520, 640), (60, 300, 999), (70, 300, 999),
                                   (200, 640, 2048), (300, 260, 1003), (1000, 520, 4096)])
def test_workspaces_of_the_stated_size(m, f, k):
    """Every call on a workspace of exactly the bytes it asks for: nothing behind it is written, and what
    it held before does not matter."""
    require_gpu()
    import paper_2510_03275_amd as P
    x, dh = D.rand(1, m, k).to(F16).cuda(), D.rand(2, m, f).to(F16).cuda()
    wg, wu = (D.rand(i, f, k, scale=k ** -0.5).to(F16).cuda() for i in (3, 4))
    g, u = (D.rand(i, m, f).to(F16).cuda() for i in (5, 6))
    g8, u8 = P.int8_quantize(wg), P.int8_quantize(wu)
    x8 = P.int8_quantize(x)
    calls = [(P.sdq_int8_linear_workspace_bytes(m, f, k), lambda ws: [P.int8_linear(x, g8, workspace=ws)]),
             (P.sdq_int8_linear_workspace_bytes(m, f, k), lambda ws: [P.int8_linear(x8, g8, workspace=ws)]),
             (P.sdq_int8_gated_linear_workspace_bytes(m, f, k),
              lambda ws: [P.int8_gated_linear(x, g8, u8, workspace=ws)]),
             (P.sdq_gated_linear_workspace_bytes(m, f, k), lambda ws: [P.gated_linear(x, wg, wu, workspace=ws)]),
             (P.sdq_gated_linear_backward_workspace_bytes(m, f, k),
              lambda ws: P.gated_linear_backward(dh, x, wg, wu, g, u, workspace=ws))]
    for need, call in calls:
        want = call(None)
        for fill in (0, 255):
            buf = torch.full((need + 4096,), fill, dtype=torch.uint8, device="cuda")
            got = call(buf[:need])
            assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool((buf[need:] == fill).all())


def test_refusals_on_the_device():
    require_gpu()
    import paper_2510_03275_amd as P
    x = torch.zeros(8, 16, dtype=F16, device="cuda")
    w8 = P.int8_quantize(torch.ones(4, 16, device="cuda"))
    w = torch.zeros(4, 16, dtype=F16, device="cuda")
    h, h32 = torch.zeros(8, 4, dtype=F16, device="cuda"), torch.zeros(8, 4, device="cuda")
    for bad in (lambda: P.int8_quantize(x.t()), lambda: P.int8_quantize(x[0]), lambda: P.int8_quantize(x.double()),
                lambda: P.int8_linear(x[:, :8], w8), lambda: P.int8_linear(x, w8, accumulate=True),
                lambda: P.int8_linear(x, w8, out=h.t()), lambda: P.int8_linear(x, w8, dtype=torch.float64),
                lambda: P.int8_linear(x, w8, out=h, dtype=F32), lambda: P.int8_linear(x, P.Int8Rows(w8.q, w8.scales[:3])),
                lambda: P.int8_linear(x.cpu(), w8), lambda: P.int8_gated_linear(x, w8, P.int8_quantize(w[:3])),
                lambda: P.gated_linear(x.float(), w.float(), w.float()), lambda: P.gated_linear(x, w, w.bfloat16()),
                lambda: P.gated_linear(x, w, w, g=h), lambda: P.gated_linear(x, w, w, g=h, u=h32),
                lambda: P.gated_linear_backward(h, x, w, w, h.bfloat16(), h.bfloat16()),
                lambda: P.gated_linear_backward(h, x, w, w, h, h, accumulate=True),
                lambda: P.gated_linear_backward(h, x, w, w, h, h, dx=x[:4])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(P.SdqError):          # starts 2 bytes off
        P.int8_quantize(torch.zeros(65, dtype=F16, device="cuda")[1:].view(4, 16))
    with pytest.raises(P.SdqError):
        P.gated_linear(x, w, w, act=3)


def _ffn_step(P, t, m, f, k, seed=0):
    """Every operator on one workspace each: the outputs of a feed-forward step and its gradients."""
    x = D.rand(seed, m, k).to(t).cuda()
    wg, wu = (D.rand(seed + i, f, k, scale=k ** -0.5).to(t).cuda() for i in (1, 2))
    g8, u8 = P.int8_quantize(wg), P.int8_quantize(wu)
    d8 = P.int8_quantize(D.rand(seed + 3, k, f, scale=f ** -0.5).float().cuda())
    g, u = torch.empty(m, f, dtype=t, device="cuda"), torch.empty(m, f, dtype=t, device="cuda")
    dh = D.rand(seed + 4, m, f).to(t).cuda()

    def step():
        h = P.gated_linear(x, wg, wu, P.SDQ_ACT_SILU, g=g, u=u)
        dx, dg, du = P.gated_linear_backward(dh, x, wg, wu, g, u)
        y = P.int8_linear(P.int8_gated_linear(P.int8_quantize(x), g8, u8, dtype=t), d8)
        return [h, dx, dg, du, y]
    return step


@pytest.mark.parametrize("m,f,k", [(1, 200, 328), (12, 264, 520), (40, 513, 72), (700, 520, 640)])
def test_graph_replays_match_eager(m, f, k):
    """Two captured graphs of the whole step, replayed in turn between eager calls."""
    require_gpu()
    import paper_2510_03275_amd as P
    steps = [_ffn_step(P, t, m, f, k, seed) for t, seed in ((F16, 1), (BF16, 9))]
    eager = [[v.clone() for v in s()] for s in steps]
    graphs = []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = s()
        graphs.append((g, out))
    for rep in range(4):
        for (g, out), want, s in zip(graphs, eager, steps):
            for o in out:
                o.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), rep
            assert all(torch.equal(a, b) for a, b in zip(s(), want)), rep
        torch.cuda.synchronize()


@pytest.mark.parametrize("m,f,k", [(2, 1000, 4096), (50, 1000, 8192), (130, 2000, 4096), (2100, 4200, 2048)])
def test_every_run_gives_the_same_bits(m, f, k):
    """Long depths on every kernel and tile height, twenty times with other work between."""
    require_gpu()
    import paper_2510_03275_amd as P
    step = _ffn_step(P, BF16, m, f, k)
    want = [v.clone() for v in step()]
    for rep in range(20):
        torch.empty(1 << 26, dtype=torch.uint8, device="cuda").fill_(rep)
        assert all(torch.equal(a, b) for a, b in zip(step(), want)), rep


@pytest.mark.parametrize("m", [1, 30, 300])
def test_graphs_share_a_workspace(m):
    """Two graphs captured on one workspace, replayed in turn on one stream, with eager calls on it between."""
    require_gpu()
    import paper_2510_03275_amd as P
    f, k = 520, 264
    ws = torch.empty(max(P.sdq_int8_gated_linear_workspace_bytes(m, f, k),
                         P.sdq_gated_linear_backward_workspace_bytes(m, f, k)), dtype=torch.uint8, device="cuda")
    wg, wu = (D.rand(i, f, k, scale=k ** -0.5).to(BF16).cuda() for i in (2, 3))
    g8, u8 = P.int8_quantize(wg), P.int8_quantize(wu)
    x, dh = D.rand(1, m, k).to(BF16).cuda(), D.rand(4, m, f).to(BF16).cuda()
    g, u = (D.rand(i, m, f).to(BF16).cuda() for i in (5, 6))
    first = lambda: [P.int8_gated_linear(x, g8, u8, workspace=ws), P.gated_linear(x, wg, wu, workspace=ws)]
    second = lambda: list(P.gated_linear_backward(dh, x, wg, wu, g, u, workspace=ws))
    want = [[v.clone() for v in c()] for c in (first, second)]
    graphs = []
    for call in (first, second):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for rep in range(3):
        for (graph, out), w, call in zip(graphs, want, (second, first)):
            for o in out:
                o.fill_(float("nan"))
            ws.fill_(255)
            graph.replay()
            call()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, w)), rep


def test_beyond_two_to_the_31_elements():
    """h, its gradient and the block's own of 2.2e9 elements each: the last rows and columns come out right."""
    require_gpu()
    import paper_2510_03275_amd as P
    m, f, k = 66000, 33000, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(m, k, generator=gen, device="cuda", dtype=BF16)
    wg, wu = (torch.randn(f, k, generator=gen, device="cuda", dtype=BF16) * 0.125 for _ in range(2))
    g, u = (torch.empty(m, f, dtype=BF16, device="cuda") for _ in range(2))
    h = P.gated_linear(x, wg, wu, g=g, u=u)
    rows, cols = [0, 32600, m - 1], [0, 17000, f - 1]
    gr, ur, eg, eu = D.gated_ref(x[rows].cpu(), wg.cpu(), wu.cpu(), 0)
    D.assert_close(h[rows], *D.gated_bound(gr, ur, eg, eu, 0, BF16))
    dh = torch.randn(m, f, generator=gen, device="cuda", dtype=BF16)
    dx, dg, du = P.gated_linear_backward(dh, x, wg, wu, g, u)
    ref = D.backward_ref(dh[rows].cpu(), x[rows].cpu(), wg.cpu(), wu.cpu(), g[rows].cpu(), u[rows].cpu(), 0, BF16)
    D.assert_close(dx[rows], *ref[0], "dx")
    # the gradients of some rows of the weights: sums over every token
    ref = D.backward_ref(dh[:, cols].cpu(), x.cpu(), wg[cols].cpu(), wu[cols].cpu(), g[:, cols].cpu(), u[:, cols].cpu(),
                         0, BF16)
    D.assert_close(dg[cols], *ref[1], "dgate")
    D.assert_close(du[cols], *ref[2], "dup")
    del dh, dx, dg, du, g, u
    # the same rows through 8 bits, against the product of the last ones alone
    w8 = P.int8_quantize(wg)
    y = P.int8_linear(x, w8, out=h)
    last = P.int8_linear(x[m - 200:].contiguous(), w8)
    assert torch.equal(y[m - 200:], last)


def test_rows_beyond_two_to_the_20():
    """More rows than one launch has workgroups."""
    require_gpu()
    import paper_2510_03275_amd as P
    m = (1 << 20) + 300
    for k in (3, 1100):       # a wave and a workgroup to a row
        x = torch.randn(m if k > 100 else 4 * m, k, device="cuda", dtype=F16)
        r = P.int8_quantize(x)
        part = P.int8_quantize(x[-500:].clone())      # a copy starts aligned
        assert torch.equal(r.q[-500:], part.q) and torch.equal(r.scales[-500:], part.scales)


@pytest.mark.parametrize("m", [3, 90])
def test_other_stream(m):
    """Calls handed a stream, while the current one works with the same allocator; two streams at once."""
    require_gpu()
    import paper_2510_03275_amd as P
    f, k = 300, 512
    x = D.rand(1, m, k).to(BF16).cuda()
    wg, wu = (D.rand(i, f, k, scale=0.05).to(BF16).cuda() for i in (2, 3))
    w8 = P.int8_quantize(wg)
    want = P.gated_linear(x, wg, wu), P.int8_linear(x, w8), P.int8_gated_linear(x, w8, w8)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for rep in range(8):
        for s in streams:
            got.append((P.gated_linear(x, wg, wu, stream=s), P.int8_linear(x, w8, stream=s),
                        P.int8_gated_linear(x, w8, w8, stream=s)))
            torch.empty(1 << 20, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_feed_forward_mixed():
    """As a model runs them: gated block -> Sigma-Delta down projection, and the 8-bit feed-forward,
    against the 64-bit block with the weights that each one stands for."""
    require_gpu()
    import paper_2510_03275_amd as P
    from oracle import linear as OL
    import oracle
    m, f, k = 9, 768, 256
    x = D.rand(1, m, k).to(F16)
    wg, wu = (D.rand(i, f, k, scale=k ** -0.5).to(F16) for i in (2, 3))
    wd = D.rand(4, k, f, scale=f ** -0.5).float()
    h = P.gated_linear(x.cuda(), wg.cuda(), wu.cuda())
    enc = P.quantize(wd.cuda(), 2.0, 3)
    y = P.linear(h, enc).cpu().double()
    ref = oracle.encode(wd.numpy(), 2.0, 3)
    want = torch.from_numpy(OL.linear_fp64(h.cpu().double().numpy(), ref.codes, ref.scales, 256, ref.m_up))
    assert float(((y - want).abs().amax(1) / want.abs().amax(1)).max()) <= 1e-3
    # 8 bits: every stage from the stage before it
    g8, u8, d8 = P.int8_quantize(wg.cuda()), P.int8_quantize(wu.cuda()), P.int8_quantize(wd.cuda())
    h8 = P.int8_gated_linear(x.cuda(), g8, u8)
    y8 = P.int8_linear(h8, d8)
    q, s = D.quantize_ref(h8.cpu())
    want = D.int8_ref(q, s, d8.q.cpu(), d8.scales.cpu())
    D.assert_close(y8, want, (D.half(F16) + 2.0 ** -22) * want.abs() + D.floor(F16))
    # and the 8-bit block near the dense one: a code is off by half a step of 1/127 of its row's
    # largest at most, so g and u by (sum |x| s_w + |w| s_x) / 2 + k s_w s_x / 4
    xd, gd, ud = x.double(), wg.double(), wu.double()
    sx = D.quantize_ref(x)[1].double()[:, None]
    err = lambda w, r: 0.5 * (xd.abs().sum(1, keepdim=True) * r.scales.cpu().double()
                              + sx * w.abs().sum(1)) + k * sx * r.scales.cpu().double() / 4
    hd, bound = D.gated_bound(xd @ gd.t(), xd @ ud.t(), err(gd, g8), err(ud, u8), 0, F16)
    D.assert_close(h8, hd, bound)


def test_gradients_against_differences():
    """The gradients of a small block against central differences of the 64-bit formula."""
    require_gpu()
    import paper_2510_03275_amd as P
    m, f, k, t = 6, 10, 12, F16
    for act in (0, 1):
        x, wg, wu = D.rand(1, m, k).to(t), D.rand(2, f, k, scale=0.5).to(t), D.rand(3, f, k, scale=0.5).to(t)
        dh = D.rand(4, m, f).to(t)
        g, u = (torch.empty(m, f, dtype=t, device="cuda") for _ in range(2))
        P.gated_linear(x.cuda(), wg.cuda(), wu.cuda(), act, g=g, u=u)
        got = P.gated_linear_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), g, u, act)
        vals = [v.double() for v in (x, wg, wu)]

        def loss(vs):
            a, _ = D.act_ref(vs[0] @ vs[1].t(), act)
            return float((dh.double() * a * (vs[0] @ vs[2].t())).sum())
        for i in range(3):
            num = torch.zeros_like(vals[i])
            for e in range(num.numel()):
                plus, minus = ([v.clone() for v in vals] for _ in range(2))
                plus[i].view(-1)[e] += 1e-5
                minus[i].view(-1)[e] -= 1e-5
                num.view(-1)[e] = (loss(plus) - loss(minus)) / 2e-5
            # g, u, dg, du and the result are rounded once each, two sums of up to 20 terms: 64 half steps
            scale = float(num.abs().max())
            assert float((got[i].cpu().double() - num).abs().max()) <= 64 * D.half(t) * scale
