"""Rotary positions with several axes against the formula in 64 bits.  Rows have three roundings, the products' and the sum's (2^-24 of the
pair's length each), and those of cosine and sine (2 half steps): 6 * 2^-24 of a pair's length; a result rounded to bf16 half a step more,
2^-8."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fs():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2302_00787_amd import binding
    binding.lib()
    return binding


def turned(x, freqs, axis_of, places, interleaved, amplitude, back):
    """x [B,H,L,d], places [axes,B,L]: 64 bits, host."""
    import torch
    r = freqs.shape[0]
    angle = torch.zeros((*places.shape[1:], r), dtype=torch.float64)
    for p in range(r):
        a = int(axis_of[p])
        if 0 <= a < places.shape[0]:
            angle[..., p] = places[a].double() * freqs[p]
    c, s = amplitude * torch.cos(angle)[:, None], amplitude * torch.sin(angle)[:, None]
    s = -s if back else s
    y = x.clone()
    i = torch.arange(r)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, r + i)
    y[..., first], y[..., second] = x[..., first] * c - x[..., second] * s, x[..., second] * c + x[..., first] * s
    return y


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,H,H2,L,d,pairs,order", [(2, 4, 2, 33, 64, [16, 8, 8], "blocks"), (1, 2, 0, 1, 32, [4, 5, 6], "cyclic"), (3, 1, 3, 7, 128, [48], "blocks"),
                                                     (1, 3, 1, 300, 80, [8, 8], "cyclic"), (2, 2, 2, 5, 24, [3, 3, 3, 2], "cyclic"), (1, 1, 1, 9, 1024, [512], "blocks"),
                                                     (1, 1, 0, 64, 8, [1], "blocks")])
def test_rows(fs, dtype, interleaved, B, H, H2, L, d, pairs, order):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(d + L)
    freqs, axis_of = fs.rotary_sections(pairs, order=order)
    places = torch.randint(-(1 << 20), 1 << 20, (len(pairs), B, L), generator=gen, dtype=torch.int32)
    rot = fs.RotaryAxes(freqs, axis_of, places.cuda(), interleaved, 1.25)
    X, X2 = (torch.randn((B, h, L, d), generator=gen).to(dt).cuda() for h in (H, max(H2, 1)))
    tol = 6 * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    for back in (False, True):
        got = fs.rotary(X, rot, X2 if H2 else None, transposed=back)
        for x, y in zip((X, X2), got if H2 else (got,)):
            want = turned(x.double().cpu(), freqs.cpu(), axis_of.cpu(), places, interleaved, 1.25, back)
            length = 1.25 * x.double().cpu().abs().amax(-1, keepdim=True) * math.sqrt(2.0)
            assert ((y.double().cpu() - want).abs() <= tol * torch.maximum(length, want.abs())).all()
    again = X.clone()
    assert fs.rotary(again, rot, out=again) is again                      # in place
    assert torch.equal(again, fs.rotary(X, rot))


@pytest.mark.parametrize("pairs,order", [([2, 3, 1, 4, 5, 1], "cyclic"), ([4] * 8, "blocks"), ([0, 3, 0, 0, 2, 0, 0, 3], "cyclic")])
def test_many_axes(fs, pairs, order):
    import torch
    gen = torch.Generator().manual_seed(sum(pairs))
    freqs, axis_of = fs.rotary_sections(pairs, order=order)
    places = torch.randint(0, 1 << 16, (len(pairs), 2, 37), generator=gen, dtype=torch.int32)
    x = torch.randn((2, 3, 37, 64), generator=gen)
    got = fs.rotary(x.cuda(), fs.RotaryAxes(freqs, axis_of, places.cuda()))
    want = turned(x.double(), freqs.cpu(), axis_of.cpu(), places, False, 1.0, False)
    length = x.double().abs().amax(-1, keepdim=True) * math.sqrt(2.0)
    assert ((got.double().cpu() - want).abs() <= 6 * 2.0 ** -24 * torch.maximum(length, want.abs())).all()


def test_one_axis_and_equal_axes_are_plain_positions(fs):
    """Bit for bit: a text's rows, whose positions are the same on all axes, are turned as by plain positions."""
    import torch
    gen = torch.Generator().manual_seed(1)
    X = torch.randn((2, 3, 50, 64), generator=gen).cuda()
    places = torch.randint(0, 100000, (2, 50), generator=gen, dtype=torch.int32).cuda()
    freqs, axis_of = fs.rotary_sections([12, 10, 10], order="cyclic", whole=True)
    want = fs.rotary(X, fs.Rotary(freqs, places))
    assert torch.equal(fs.rotary(X, fs.RotaryAxes(freqs, axis_of, places.expand(3, 2, 50))), want)
    assert torch.equal(fs.rotary(X, fs.RotaryAxes(freqs, torch.zeros_like(axis_of), places[None])), want)
    shared = fs.rotary(X, fs.RotaryAxes(freqs, axis_of, places[:1].expand(3, 50)))
    assert torch.equal(shared, fs.rotary(X, fs.Rotary(freqs, places[0])))


def test_pairs_of_no_axis_and_strides(fs):
    """axis_of beyond the axes: position 0 (no reading there); positions and rows with strides of their own."""
    import torch
    gen = torch.Generator().manual_seed(2)
    freqs, axis_of = fs.rotary_sections([8, 8])
    axis_of[3], axis_of[9] = -1, 2
    table = torch.randint(0, 5000, (4, 40, 2, 3), generator=gen, dtype=torch.int32).cuda()
    places = table[::2, 1::2, :, 1].permute(2, 0, 1)                       # [2 axes, 2 sequences, 20 rows]
    X = torch.randn((2, 20, 3, 40), generator=gen).cuda().transpose(1, 2)
    got = fs.rotary(X, fs.RotaryAxes(freqs, axis_of, places))
    want = turned(X.double().cpu(), freqs.cpu(), axis_of.cpu(), places.cpu(), False, 1.0, False)
    assert (got.double().cpu() - want).abs().max() <= 6 * 2.0 ** -24 * 2 * X.abs().max().item()


def test_captured(fs):
    import torch
    gen = torch.Generator().manual_seed(3)
    freqs, axis_of = fs.rotary_sections([16, 8, 8])
    X, places = torch.randn((1, 4, 100, 64), generator=gen).bfloat16().cuda(), torch.zeros((3, 100), dtype=torch.int32, device="cuda")
    rot = fs.RotaryAxes(freqs, axis_of, places)
    fs.rotary(X, rot)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fs.rotary(X, rot)
    for i in range(3):
        places.copy_(torch.randint(0, 1000, (3, 100), generator=gen, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, fs.rotary(X, rot))


def test_a_head_that_forgets_on_turned_rows(fs):
    """Together, as in a layer over clips and text: rows turned, attended, gradients turned back; then a token that goes on from the state.
    Against the formulas in 64 bits; fp32 rows, so that the parts' roundings are those of their tests."""
    import torch
    from .test_gpu_decay import F32, backward, close, forward
    gen = torch.Generator().manual_seed(4)
    B, H, Hk, L, d, dv, s = 2, 4, 2, 150, 64, 32, 0.125
    freqs, axis_of = fs.rotary_sections([16, 8, 8])
    places = torch.stack([torch.arange(L + 1) // 24, torch.arange(L + 1) // 6 % 4, torch.arange(L + 1) % 6]).to(torch.int32)
    Q, K, V, dY = (torch.randn((B, h, L + 1, w), generator=gen).cuda() for h, w in ((H, d), (Hk, d), (Hk, dv), (H, dv)))
    g = torch.tensor([-0.02, -0.3])
    rows, last = fs.RotaryAxes(freqs, axis_of, places[:, :L].cuda()), fs.RotaryAxes(freqs, axis_of, places[:, L:].cuda())
    pool = fs.decay_state_new(B, Hk, d, dv)
    q, k = fs.rotary(Q[:, :, :L], rows, K[:, :, :L])
    Y = fs.decay_attention(q, k, V[:, :, :L], g.cuda(), s, after=pool)
    dq, dk, dv_, _ = fs.decay_attention_backward(q, k, V[:, :, :L], dY[:, :, :L], g.cuda(), s)
    dQ, dK = fs.rotary(dq, rows, dk, transposed=True)
    q1, k1 = fs.rotary(Q[:, :, L:], last, K[:, :, L:])
    y = fs.decay_step(pool, q1, k1, V[:, :, L:], g.cuda(), s)
    at = places[:, None].expand(3, B, L + 1)
    tq, tk = (turned(x.double().cpu(), freqs.cpu(), axis_of.cpu(), at, False, 1.0, False) for x in (Q, K))
    for b in range(B):
        v, dy = V[b].double().cpu(), dY[b].double().cpu()
        want, S = forward(tq[b], tk[b], v, g.double(), s, torch.zeros(Hk, d, dv, dtype=torch.float64), L + 1)
        close(torch.cat([Y[b], y[b]], 1), want, F32)
        close(pool[b], S, F32)
        zero = torch.zeros_like(S)
        gq, gk, gv, _ = backward(tq[b, :, :L], tk[b, :, :L], v[:, :L], dy[:, :L], g.double(), s, zero, zero, L)
        gq, gk = (turned(x[None], freqs.cpu(), axis_of.cpu(), at[:, :1, :L], False, 1.0, True)[0] for x in (gq, gk))
        for x, w in zip((dQ[b], dK[b], dv_[b]), (gq, gk, gv)):
            close(x, w, F32)
