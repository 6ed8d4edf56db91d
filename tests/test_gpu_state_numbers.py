"""Numbers that kept states meet besides the everyday ones, against the formulas in 64 bits of test_gpu_state.

Values with a mean.  dq is s sum_m p_m (dY . T_m - delta z_m) W_m, dk s sum_m S_m (V . dT_m + dz_m) W_m and s^2 sum_m S_m (V . dT_m + dz_m) times (C2 + C2') k:
where values share a mean, the two terms of each bracket are far larger than their difference.  The products are fp32's: a term is off by a
few roundings of 2^-24 of itself, each in its own direction, sums over m by a few more; sixteen of them, 2^-20 of the root of the terms' sum of
squares (`parts`), is the bar.  Two bf16 pieces of a factor would be off by up to 2^-17 of it.  A result rounded to bf16 is off by up to half a step, 2^-8 of
the power of two below it, and so by 2^-8 / sqrt(3) of the norm; features are off by GRAD (test_gpu_state).
"""
import math

import pytest

from .test_gpu_state import F32, GRAD, check, make_theta, rows, turned
from .test_gpu_state_shares import fs, oracle, parts_of  # noqa: F401 (fs: a fixture)

pytestmark = pytest.mark.gpu

ROUNDED = 2.0 ** -8 / math.sqrt(3.0)


@pytest.mark.parametrize("d,dv,M,B,heads,L,Lk,turn", [
    (64, 64, 256, 2, 2, 512, 300, False), (64, 64, 256, 8, 8, 70, 90, False), (64, 64, 96, 8, 8, 40, 60, True), (64, 64, 96, 2, 1, 90, 200, True),
    (128, 128, 512, 2, 2, 100, 130, False), (128, 128, 64, 8, 8, 40, 50, True), (32, 32, 64, 8, 8, 40, 70, False), (32, 32, 64, 2, 2, 300, 200, True),
    (48, 40, 100, 8, 8, 40, 50, False), (96, 128, 70, 2, 1, 80, 100, True)])
def test_gradients_of_values_with_a_mean(fs, d, dv, M, B, heads, L, Lk, turn):  # noqa: F811
    import torch
    gen, s, dt = torch.Generator().manual_seed(d + M + L), d ** -0.25, torch.bfloat16
    theta, omega = make_theta(gen, "iso", heads, d), torch.randn((heads, M, d), generator=gen)
    o, f = oracle(theta, omega, s, heads), fs.state_prepare(theta.cuda(), omega.cuda(), s)
    K, V, Q, dY = (rows(gen, torch.float32, B, heads, n, c) for n, c in ((Lk, d), (Lk, dv), (L, d), (L, dv)))
    K, V, Q, dY = K.to(dt), (V + 128).to(dt), Q.to(dt), (dY + 1).to(dt)
    rot = fs.Rotary(fs.rotary_frequencies(d // 16 * 16)) if turn else None
    k64, q64 = (turned(x.double().cpu(), rot).cuda() for x in (K, Q))
    state = fs.state_append(f, fs.state_new(B, heads, M, dv), K, V, rotary=rot, fresh=True)
    Y = fs.state_attention(f, state, Q, rotary=rot)
    dQ, ds = fs.state_attention_backward(f, state, Q, dY, rotary=rot)
    dK, dV = fs.state_append_backward(f, state, ds, K, V, rotary=rot)
    want = [torch.empty(t.shape, dtype=torch.float64, device="cuda") for t in (Y, dQ, dK, dV)]
    parts = [0.0] * 4                            # sums of their squares
    for b in range(B):
        for h in range(heads):
            T, z, shift = state.T[b, h].double(), state.z[b, h].double(), state.shift[b, h].double()
            q, k, v, dy, dT, dz = q64[b, h], k64[b, h], V[b, h].double(), dY[b, h].double(), ds.T[b, h].double(), ds.z[b, h].double()
            want[0][b, h] = o.read((T, z, None), h, q)
            want[1][b, h] = o.read_backward((T, z, None), h, q, dy)[0]
            want[2][b, h], want[3][b, h] = o.append_backward(shift, h, k, v, dT, dz)
            e = s * q @ o.W1[h].T + o.bias[h]
            p = torch.exp(e - e.max(1, keepdim=True).values)
            p = p / (p @ z)[:, None]
            delta = ((p @ T) * dy).sum(1, keepdim=True)
            parts[1] += float(s * s * ((p * ((dy @ T.T).abs() + delta.abs() * z)).square() @ o.W1[h].square()).sum())
            u = (torch.exp(o.key_exponents(h, k) - shift * math.log(2)) * ((v @ dT.T).abs() + dz.abs())).square()
            parts[2] += float((s * s * u @ o.W2[h].square() + s ** 4 * u.sum(1, keepdim=True) * (k @ (o.C2[h] + o.C2[h].T)).square()).sum())
    if rot is not None:
        want[1], want[2] = (turned(x.cpu(), rot, transposed=True).cuda() for x in want[1:3])
    for name, got, ref, part, tol in zip(("Y", "dQ", "dK", "dV"), (Y, dQ, dK, dV), want, parts, (F32, GRAD, GRAD, F32)):
        off, norm = float((got.double() - ref).norm()), float(ref.norm())
        assert off <= (ROUNDED + tol) * norm + 2.0 ** -20 * math.sqrt(part), (name, off / norm, math.sqrt(part) / norm)


@pytest.mark.parametrize("d,dv,M,heads,group,L", [(64, 64, 256, 1, 1, 20), (64, 64, 96, 1, 2, 9000), (128, 128, 300, 2, 1, 33), (128, 100, 64, 1, 1, 17000),
                                                   (32, 32, 64, 1, 3, 40), (20, 32, 70, 2, 1, 6000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power", [-70, -135])
def test_rows_that_read_what_a_state_holds_little_of(fs, d, dv, M, heads, group, L, dtype, power):  # noqa: F811
    """States whose T and z are 2^power where rows peak: everywhere (the first sequence's), or for one row of many (the second's).  Normalisers of 2^power of
    a row's largest feature, below the smallest normal number at -135, have quotients and gradients like any others; the tolerances are the usual ones
    (T and z are what the state holds, rounded or not).  dY is 2^-30, so that the gradients of T, 2^(-power - 30), are numbers."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen, s = torch.Generator().manual_seed(d + M + L), d ** -0.25
    theta, omega = make_theta(gen, "iso", heads, d), torch.randn((heads, M, d), generator=gen)
    o, f = oracle(theta, omega, s, heads), fs.state_prepare(theta.cuda(), omega.cuda(), s)
    H = heads * group
    Q, dY = rows(gen, dt, 2, H, L, d), rows(gen, dt, 2, H, L, dv, scale=2.0 ** -30)
    Q[1, :, 3] *= 6
    state = fs.state_new(2, heads, M, dv)
    state.T.copy_(torch.randn(state.T.shape, generator=gen))
    state.z.copy_(0.5 + torch.rand(state.z.shape, generator=gen))
    state.shift.zero_()
    for h in range(heads):
        e = (s * Q[1, h * group, 3].double() @ o.W1[h].T + o.bias[h]) / math.log(2.0)
        less = (power - (e - e.max())).clamp(max=0.0)          # every feature adds as much to that row, or less, as the largest
        for t, scale in ((state.T, torch.exp2(less)[:, None]), (state.z, torch.exp2(less))):
            t[0, h] = (t[0, h].double() * 2.0 ** power).float()
            t[1, h] = (t[1, h].double() * scale).float()
    unread = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = fs.state_attention(f, state, Q, unread=unread)
    dQ, ds = fs.state_attention_backward(f, state, Q, dY)
    assert int(unread) == 0
    for b in range(2):
        for h in range(heads):
            st = (state.T[b, h].double(), state.z[b, h].double(), None)
            dT, dz = torch.zeros_like(st[0]), torch.zeros_like(st[1])
            for i in range(h * group, (h + 1) * group):
                check(Y[b, i], o.read(st, h, Q[b, i].double()).cpu(), F32, "Y")
                dq, t, z = o.read_backward(st, h, Q[b, i].double(), dY[b, i].double())
                dT, dz = dT + t, dz + z
                # (dy is of the outputs' size times 2^-30: the two parts of dq as in test_gpu_state_shares)
                check(dQ[b, i], dq.cpu(), GRAD, "dQ", parts_of(o, st, h, dY[b, i].double()).cpu())
            check(ds.T[b, h].reshape(1, -1), dT.reshape(1, -1).cpu(), F32, "dT")
            check(ds.z[b, h][None], dz[None].cpu(), GRAD, "dz")


@pytest.mark.parametrize("B,heads,L,M,d,dtype", [(2, 1, 1, 64, 64, "f32"), (3, 2, 40, 64, 64, "bf16"), (2, 2, 700, 256, 64, "bf16"), (2, 1, 300, 100, 48, "f32"),
                                                 (260, 1, 5, 32, 16, "f32"), (2, 1, 90, 512, 128, "bf16")])
def test_a_key_that_is_not_a_number_shows_in_its_state(fs, B, heads, L, M, d, dtype):  # noqa: F811
    """All of that state, and no other; appended to an empty state and to one with keys, as a sequence's only keys, among others and as a token."""
    import torch
    dt, nan = torch.bfloat16 if dtype == "bf16" else torch.float32, float("nan")
    gen, s = torch.Generator().manual_seed(B + L), d ** -0.25
    theta, omega = make_theta(gen, "iso", heads, d), torch.randn((heads, M, d), generator=gen)
    f = fs.state_prepare(theta.cuda(), omega.cuda(), s)
    K, V, q = (rows(gen, dt, B, heads, n, d) for n in (L, L, 1))
    h = heads - 1
    for first, last in ((0, L), (L // 2, L // 2 + 1)):
        bad = K.clone()
        bad[1, h, first:last, d // 2] = nan
        for fresh in (True, False):
            state = fs.state_append(f, fs.state_new(B, heads, M, d), K, V)
            good = fs.state_append(f, fs.state_append(f, fs.state_new(B, heads, M, d), K, V), K, V, fresh=fresh)
            fs.state_append(f, state, bad, V, fresh=fresh)
            for t, g in zip(state, good):
                assert t[1, h].isnan().all()
                t[1, h] = g[1, h]
                assert torch.equal(t, g)
    # a token onto an empty state and onto one with keys; then a good one, and good keys
    k, v = K[:, :, :1], V[:, :, :1]
    bad = k.clone()
    bad[1, h, 0, 0] = nan
    for state in (fs.state_new(B, heads, M, d), fs.state_append(f, fs.state_new(B, heads, M, d), K, V)):
        good = fs.State(*(t.clone() for t in state))
        for key in (bad, k):
            Y, Yg = fs.state_step(f, state, q, key, v), fs.state_step(f, good, q, k, v)
            assert Y[1, h].isnan().all() and all(t[1, h].isnan().all() for t in state)
            Y[1, h] = Yg[1, h]
            assert torch.equal(Y, Yg)
        fs.state_append(f, state, K, V)
        fs.state_append(f, good, K, V)
        for t, g in zip(state, good):
            assert t[1, h].isnan().all()
            t[1, h] = g[1, h]
            assert torch.equal(t, g)
    # a query: its row, and the gradient of what it read
    state = fs.state_append(f, fs.state_new(B, heads, M, d), K, V)
    for n in (1, L):
        Q, dY = rows(gen, dt, B, heads, n, d), rows(gen, dt, B, heads, n, d)
        Yg, (dQg, dg) = fs.state_attention(f, state, Q), fs.state_attention_backward(f, state, Q, dY)
        Q[1, h, n // 2, 0] = nan
        Y, (dQ, ds) = fs.state_attention(f, state, Q), fs.state_attention_backward(f, state, Q, dY)
        for t, g in ((Y, Yg), (dQ, dQg)):
            assert t[1, h, n // 2].isnan().all()
            t[1, h, n // 2] = g[1, h, n // 2]
            assert torch.equal(t, g)
        for t, g in ((ds.T, dg.T), (ds.z, dg.z)):
            assert t[1, h].isnan().all()
            t[1, h] = g[1, h]
            assert torch.equal(t, g)


@pytest.mark.parametrize("B,slots,heads", [(3000, 2500, 1), (2600, 1, 2), (1500, 3, 1), (300, 5, 1), (1025, 1, 1)])
def test_gradients_of_states_with_many_readers(fs, B, slots, heads):  # noqa: F811
    """Readers of a slot anywhere among thousands of sequences, and thousands of readers of one slot; some sequences have none."""
    import torch
    gen, d, M, L = torch.Generator().manual_seed(B), 16, 32, 2
    s = d ** -0.25
    theta, omega = make_theta(gen, "iso", heads, d), torch.randn((heads, M, d), generator=gen)
    o, f = oracle(theta, omega, s, heads), fs.state_prepare(theta.cuda(), omega.cuda(), s)
    where = torch.randint(-1, slots + 1, (B,), generator=gen).to(torch.int32)
    Q, dY = (rows(gen, torch.float32, B, heads, L, d) for _ in range(2))
    state = fs.state_new(slots, heads, M, d)
    state.T.copy_(torch.randn(state.T.shape, generator=gen))
    state.z.copy_(0.5 + torch.rand(state.z.shape, generator=gen))
    state.shift.zero_()
    dQ, ds = fs.state_attention_backward(f, state, Q, dY, slots=where.cuda())
    for h in range(heads):
        e = s * Q[:, h].double() @ o.W1[h].T + o.bias[h]
        p = torch.exp(e - e.amax(2, keepdim=True))
        at = where.long().clamp(0, slots - 1).cuda()
        z, T, dy = state.z[at, h].double()[:, None], state.T[at, h].double(), dY[:, h].double()
        p = p / (p * z).sum(2, keepdim=True)
        delta = (torch.bmm(p, T) * dy).sum(2, keepdim=True)
        gT, gz = torch.bmm(p.transpose(1, 2).contiguous(), dy), -(p * delta).sum(1)
        there = ((where >= 0) & (where < slots)).cuda().double()
        dT = torch.zeros_like(state.T[:, h], dtype=torch.float64).index_add_(0, at, gT * there[:, None, None])
        dz = torch.zeros_like(state.z[:, h], dtype=torch.float64).index_add_(0, at, gz * there[:, None])
        check(ds.T[:, h].reshape(1, -1), dT.reshape(1, -1).cpu(), F32, "dT")
        check(ds.z[:, h].reshape(1, -1), dz.reshape(1, -1).cpu(), GRAD, "dz")
    again = fs.state_attention_backward(f, state, Q, dY, slots=where.cuda())[1]
    assert torch.equal(again.T, ds.T) and torch.equal(again.z, ds.z)


def test_angles_lose_nothing_before_cosine_and_sine(fs):  # noqa: F811
    """Rows (1, 0) turned: cosine and sine themselves.  Each is off by a step of numbers below 1, 2^-24, at most, and by the half step of the sum
    with what the angle had below 32 bits."""
    import torch
    n, L = 128, 4096
    rot = fs.Rotary(fs.rotary_frequencies(n), torch.arange(L, dtype=torch.int32, device="cuda") * 31)
    x = torch.zeros((1, 1, L, n), device="cuda")
    x[..., : n // 2] = 1
    y = fs.rotary(x, rot).double().cpu()[0, 0]
    ang = rot.positions.cpu().double()[:, None] * rot.freqs.cpu()
    want = torch.cat([torch.cos(ang), torch.sin(ang)], dim=1)
    assert float((y - want).abs().max()) <= 1.5 * 2.0 ** -24


@pytest.mark.parametrize("B,heads,group,d,dv,M", [(4, 2, 1, 64, 64, 256), (4, 1, 1, 32, 30, 64), (6, 1, 4, 128, 128, 300), (300, 1, 1, 64, 40, 256), (4, 2, 5, 48, 48, 512)])
@pytest.mark.parametrize("power", [-70, -135])
def test_tokens_that_read_what_a_state_holds_little_of(fs, B, heads, group, d, dv, M, power):  # noqa: F811
    """As above, for tokens: in one launch and in two.  The states' shift is 300, so that the new key adds nothing (it is 2^-300 of them)."""
    import torch
    gen, s = torch.Generator().manual_seed(B + d), d ** -0.25
    theta, omega = make_theta(gen, "iso", heads, d), torch.randn((heads, M, d), generator=gen)
    o, f = oracle(theta, omega, s, heads), fs.state_prepare(theta.cuda(), omega.cuda(), s)
    q, k, v = (rows(gen, torch.float32, B, *n) for n in ((heads * group, 1, d), (heads, 1, d), (heads, 1, dv)))
    q[1::2] *= 6
    state = fs.state_new(B, heads, M, dv)
    state.T.copy_(torch.randn(state.T.shape, generator=gen))
    state.z.copy_(0.5 + torch.rand(state.z.shape, generator=gen))
    state.shift.fill_(300.0)
    for b in range(B):
        for h in range(heads):
            less = torch.full((M,), float(power), dtype=torch.float64, device="cuda")
            if b % 2:
                e = (s * q[b, h * group, 0].double() @ o.W1[h].T + o.bias[h]) / math.log(2.0)
                less = (power - (e - e.max())).clamp(max=0.0)
            state.T[b, h] = (state.T[b, h].double() * torch.exp2(less)[:, None]).float()
            state.z[b, h] = (state.z[b, h].double() * torch.exp2(less)).float()
    before = [t.clone() for t in state]
    unread = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = fs.state_step(f, state, q, k, v, unread=unread)
    assert int(unread) == 0 and all(torch.equal(t, g) for t, g in zip(state, before))
    for b in range(B):
        for i in range(heads * group):
            h = i // group
            check(Y[b, i], o.read((state.T[b, h].double(), state.z[b, h].double(), None), h, q[b, i].double()).cpu(), F32, "Y")
