"""Rotary positions and attention through kept states against plain formulas in 64 bits, through the public entry points.

Tolerances.  An exponent (base 2) of these inputs is at most about 60 in size and is the rounded sum of a product, a bias and a row
term: it is off by at most 4 half steps of 60, 4 * 60 * 2^-24 = 1.4e-5, and the products with it are good to 2^-22, so that a feature is
off by 1e-5 of itself at the most, by a few 1e-6 on average.  Sums of features and their products: F32 = 2e-5 of the norm; gradients
are differences of such products (dY . T - delta z), up to ten times as large as themselves: GRAD = 1e-4.  A result rounded to
bf16 is off by half a step more, 2^-8 of itself.  A single row's dq = sum p u (dY . T_m) W_m - delta sum p u z_m W_m can be far smaller than its
two parts (one feature carries the row: then W_m is the same in both), each of which is at most |dY| max |T_m / z_m| max |W_m| as sum p u z
= 1, and off by 2e-5 of that: numbers of dq are held to that size, not to their row's largest.  Rows turned by their positions have three roundings, the products' and the sum's (2^-24
of the pair's length each), and those of cosine and sine (2 half steps): 6 * 2^-24.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

F32, GRAD = 2e-5, 1e-4
HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def fs():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2302_00787_amd import binding
    binding.lib()
    return binding


# ------------------------------------------------------------------------------------------------ formulas in 64 bits
def make_theta(gen, family, groups, d):
    import torch
    a = -0.02 - 0.06 * torch.rand((groups,), generator=gen, dtype=torch.float64)
    b = torch.sqrt(1 - 4 * a)[:, None, None]
    G = inv = torch.eye(d, dtype=torch.float64).expand(groups, d, d)
    if family == "dense":
        G = G + torch.randn((groups, d, d), generator=gen, dtype=torch.float64) * (0.15 / math.sqrt(d))
        inv = torch.linalg.inv(G)
    head = torch.zeros((groups, 8), dtype=torch.float64)
    head[:, 0] = 0.25 * d * torch.log(1 - 4 * a)
    head[:, 2] = 3.0 if family == "iso" else 0.0
    parts = [head, a[:, None].expand(groups, d), b * G, b * inv.transpose(1, 2), -0.5 * G.transpose(1, 2) @ G, -0.5 * inv @ inv.transpose(1, 2)]
    return torch.cat([p.reshape(groups, -1) for p in parts], 1).float()


class Oracle:
    """W1, W2 [heads, M, d], bias [heads, M], C2 [heads, d, d], natural logarithms, for scaled rows."""

    def __init__(self, theta, omega, s, heads):
        import torch
        th, om = theta.double().expand(heads, -1), omega.double().expand(heads, -1, -1)
        M, d = om.shape[1:]
        A, B1, B2, C2 = (th[:, 8 + i:8 + j] for i, j in ((0, d), (d, d + d * d), (d + d * d, d + 2 * d * d), (d + 3 * d * d, d + 4 * d * d)))
        self.W1, self.W2 = om @ B1.reshape(heads, d, d), om @ B2.reshape(heads, d, d)
        self.bias = (om * om * A[:, None]).sum(-1) + th[:, :1] - 0.5 * math.log(M)
        self.C2, self.s, self.heads, self.M = C2.reshape(heads, d, d), s, heads, M

    def key_exponents(self, h, k):
        y = self.s * k
        return y @ self.W2[h].T + self.bias[h] + ((y @ self.C2[h]) * y).sum(1, keepdim=True)

    def append(self, state, b, h, k, v):
        """state: (T, z, shift base 2) of one sequence and head."""
        import torch
        T, z, shift = state
        if k.shape[0] == 0:
            return state
        e = self.key_exponents(h, k)
        new = torch.maximum(shift, e.max() / math.log(2))
        keep = torch.exp2(shift - new)
        S = torch.exp(e - new * math.log(2))
        return T * keep + S.T @ v, z * keep + S.sum(0), new

    def read(self, state, h, q):
        import torch
        T, z, _ = state
        e = self.s * q @ self.W1[h].T + self.bias[h]
        P = torch.exp(e - e.max(1, keepdim=True).values)
        den = P @ z
        return torch.where(den[:, None] > 0, P @ T / den[:, None], torch.zeros_like(P @ T))

    def read_backward(self, state, h, q, dy):
        import torch
        T, z, _ = state
        e = self.s * q @ self.W1[h].T + self.bias[h]
        P = torch.exp(e - e.max(1, keepdim=True).values)
        den = (P @ z)[:, None]
        P = torch.where(den > 0, P / den, torch.zeros_like(P))
        delta = ((P @ T) * dy).sum(1)
        dq = self.s * (P * (dy @ T.T - delta[:, None] * z)) @ self.W1[h]
        return dq, P.T @ dy, -(P.T @ delta)

    def append_backward(self, shift, h, k, v, dT, dz):
        import torch
        S = torch.exp(self.key_exponents(h, k) - shift * math.log(2))
        dE = S * (v @ dT.T + dz)
        dk = self.s * dE @ self.W2[h] + self.s ** 2 * dE.sum(1, keepdim=True) * (k @ (self.C2[h] + self.C2[h].T))
        return dk, S @ dT


def turned(x, rot, transposed=False):
    """[B,H,L,d] in 64 bits."""
    import torch
    if rot is None:
        return x
    B, H, L, d = x.shape
    n = 2 * rot.freqs.shape[0]
    pos = torch.arange(L) if rot.positions is None else rot.positions.cpu()
    ang = pos.double().reshape(-1, 1, L, 1) * rot.freqs.cpu()
    c, s = rot.amplitude * torch.cos(ang), rot.amplitude * torch.sin(ang) * (-1 if transposed else 1)
    y = x.clone()
    if rot.interleaved:
        u, v = x[..., 0:n:2], x[..., 1:n:2]
        y[..., 0:n:2], y[..., 1:n:2] = u * c - v * s, v * c + u * s
    else:
        u, v = x[..., :n // 2], x[..., n // 2:n]
        y[..., :n // 2], y[..., n // 2:n] = u * c - v * s, v * c + u * s
    return y


# ------------------------------------------------------------------------------------------------ helpers
def rows(gen, dt, B, H, L, d, scale=1.0, packed=False):
    """[B,H,L,d] on the GPU with rows that start at 16 bytes; packed: a view of [B,L,H,.] with numbers between the rows."""
    import torch
    q = 8 if dt == torch.bfloat16 else 4
    w = (d + q - 1) // q * q + (q if packed else 0)
    x = scale * torch.randn((B, L, H, w) if packed else (B, H, L, w), generator=gen)
    x = x.to(dt).cuda()
    x = x.transpose(1, 2) if packed else x
    return x[..., :d]


def empty_rows(dt, B, H, L, d):
    import torch
    w = (d + 7) // 8 * 8
    return torch.full((B, H, L, w), float("nan"), dtype=dt, device="cuda")[..., :d]


def check(got, ref, tol, what="", size=None):
    """Norm over everything, and number by number against the largest of the last axis (or `size` of its row)."""
    import torch
    g, r = got.double().cpu(), ref
    assert g.shape == r.shape, (what, g.shape, r.shape)
    assert torch.isfinite(g).all(), what
    half = HALF if got.dtype == torch.bfloat16 else 0.0
    err, top = (g - r).abs(), r.abs().amax(-1, keepdim=True) if size is None else size
    over = float((err - half * r.abs() - 10 * tol * top).max())
    assert over <= 1e-30, (what, over, float(top.max()))
    norm, off = float(r.norm()), float((g - r).norm())
    assert off <= (tol + half) * norm + 1e-30, (what, off, norm)


def make_rot(fs, kind, d, B, L, gen):
    import torch
    if kind is None:
        return None
    name, share = kind
    n = max(2, int(d * share) // 2 * 2)
    pos = torch.randint(0, 1 << 20, (B, 1), generator=gen) + torch.arange(L)
    return fs.Rotary(fs.rotary_frequencies(n), pos.to(torch.int32).cuda(), name == "interleaved", 1.1)


def oracle_states(o, B, slots, dv):
    import torch
    return [[(torch.zeros((o.M, dv), dtype=torch.float64), torch.zeros(o.M, dtype=torch.float64), torch.tensor(-math.inf, dtype=torch.float64))
             for _ in range(o.heads)] for _ in range(slots)]


def check_states(state, want, tol=F32):
    import torch
    for s, heads in enumerate(want):
        for h, (T, z, shift) in enumerate(heads):
            assert float(state.shift[s, h]) == float("-inf") if shift == -math.inf else abs(float(state.shift[s, h]) - float(shift)) <= 2e-5
            check(state.T[s, h].reshape(1, -1), T.reshape(1, -1), tol, ("T", s, h))
            check(state.z[s, h].reshape(1, -1), z.reshape(1, -1), tol, ("z", s, h))


SHAPES = [  # d, dv, M, heads, group, L, dtype, family, rotation
    (64, 64, 256, 2, 1, 100, "bf16", "iso", ("half", 1.0)),
    (64, 64, 256, 2, 2, 70, "bf16", "iso", None),
    (16, 16, 64, 1, 1, 33, "f32", "iso", None),
    (128, 128, 512, 1, 2, 130, "f32", "dense", ("half", 0.5)),
    (128, 128, 512, 1, 1, 65, "bf16", "dense", ("interleaved", 1.0)),
    (96, 40, 100, 2, 3, 31, "f32", "dense", ("half", 0.25)),
    (30, 63, 33, 2, 1, 40, "f32", "iso", ("half", 0.8)),
    (5, 3, 1, 1, 2, 64, "f32", "dense", None),
    (128, 16, 130, 2, 1, 1, "bf16", "iso", ("interleaved", 0.25)),
    (32, 128, 290, 1, 1, 129, "bf16", "dense", ("half", 1.0)),
    (1, 1, 32, 3, 1, 7, "f32", "iso", None),
    (80, 80, 31, 1, 4, 257, "f32", "iso", ("interleaved", 0.7)),
]


def setup(fs, shape, B, seed):
    import torch
    d, dv, M, heads, group, L, dtype, family, kind = shape
    gen = torch.Generator().manual_seed(seed)
    s = d ** -0.25
    theta, omega = make_theta(gen, family, heads, d), torch.randn((heads, M, d), generator=gen)
    o = Oracle(theta, omega, s, heads)
    f = fs.state_prepare(theta.cuda(), omega.cuda(), s)
    assert f.desc.dense_c2 == (family == "dense")
    return gen, o, f, torch.bfloat16 if dtype == "bf16" else torch.float32


# ------------------------------------------------------------------------------------------------ rotary
@pytest.mark.parametrize("d,n,interleaved", [(64, 64, False), (64, 64, True), (128, 96, True), (128, 32, False), (80, 24, False), (80, 24, True),
                                             (30, 14, False), (2, 2, True), (7, 6, True), (520, 512, False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rotary(fs, d, n, interleaved, dtype):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(d + n)
    B, H, H2, L = 3, 3, 2, 11
    X, X2 = rows(gen, dt, B, H, L, d, packed=True), rows(gen, dt, B, H2, L, d)
    pos = torch.randint(0, 2 ** 31 - 1, (B, L), generator=gen).to(torch.int32)
    pos[0, 0], pos[0, 1], pos[1, 0] = 0, 2 ** 31 - 1, -5
    rot = fs.Rotary(fs.rotary_frequencies(n), pos.cuda(), interleaved, 1.25)
    def close(got, ref):
        step = HALF if dt == torch.bfloat16 else 0.0
        size = ref.abs().amax(-1, keepdim=True) * 2 ** 0.5
        assert ((got.double().cpu() - ref).abs() <= step * ref.abs() + 6 * 2.0 ** -24 * size).all()
    for back in (False, True):
        Y, Y2 = empty_rows(dt, B, H, L, d), empty_rows(dt, B, H2, L, d)
        fs.rotary(X, rot, X2, transposed=back, out=Y, out2=Y2)
        close(Y, turned(X.double().cpu(), rot, back))
        close(Y2, turned(X2.double().cpu(), rot, back))
    # one tensor alone, positions shared or implied; in place
    one = fs.Rotary(rot.freqs, pos[1].cuda(), interleaved, 1.25)
    close(fs.rotary(X, one, out=empty_rows(dt, B, H, L, d)), turned(X.double().cpu(), one))
    want = turned(X.double().cpu(), rot._replace(positions=None))
    X = X.clone() if X.is_contiguous() else X
    close(fs.rotary(X, rot._replace(positions=None), out=X), want)


def test_rotary_long_batches_and_gradient(fs):
    """Turning back is the transpose: <R x, y> = <x, R' y>; with amplitude 1 it is the inverse.  More tokens than a workgroup."""
    import torch
    gen = torch.Generator().manual_seed(0)
    X, Y = rows(gen, torch.float32, 2, 5, 1111, 64), rows(gen, torch.float32, 2, 5, 1111, 64)
    rot = fs.Rotary(fs.rotary_frequencies(48, scaling="blend", factor=8.0, original_length=512), None, False, 1.0)
    RX, RtY = fs.rotary(X, rot), fs.rotary(Y, rot, transposed=True)
    a, b = (RX.double() * Y.double()).sum(), (X.double() * RtY.double()).sum()
    assert abs(float(a - b)) <= 1e-6 * float(X.double().norm() * Y.double().norm())
    back = fs.rotary(RX, rot, transposed=True)
    assert float((back - X).abs().max()) <= 12 * 2.0 ** -24 * float(X.abs().max()) * 2
    assert torch.equal(back[..., 48:], X[..., 48:])


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:7]))
def test_append_and_attention(fs, shape):
    """Two appends of a padded batch with NaN in the padding, a sequence without rows, one without a slot and one whose slot is taken;
    then queries of other lengths, of every sequence, some of one slot, one of an empty state."""
    import torch
    d, dv, M, heads, group, L, dtype, family, kind = shape
    B, nslots = 6, 8
    gen, o, f, dt = setup(fs, shape, B, 17 + d)
    state = fs.state_new(nslots, heads, M, dv)
    want = oracle_states(o, B, nslots, dv)
    slots = torch.tensor([5, 0, 7, -1, 0, 2], dtype=torch.int32)          # 4: the slot of 1; 3: none
    for turn in range(2):
        n = max(1, L - 9 * turn)
        K, V = rows(gen, dt, B, heads, n, d, packed=True), rows(gen, dt, B, heads, n, dv)
        lengths = torch.tensor([n, 1, 0 if turn == 0 else max(1, n // 2), n, n, n + 5], dtype=torch.int32)
        rot = make_rot(fs, kind, d, B, n, gen)
        k, v = turned(K.double().cpu(), rot), V.double().cpu()
        for b in range(B):
            m = min(int(lengths[b]), n)
            K[b, :, m:], V[b, :, m:] = float("nan"), float("inf")
            if b in (3, 4):
                continue
            for h in range(heads):
                want[int(slots[b])][h] = o.append(want[int(slots[b])][h], b, h, k[b, h, :m], v[b, h, :m])
        left = torch.zeros(1, dtype=torch.int32, device="cuda")
        fs.state_append(f, state, K, V, lengths=lengths.cuda(), slots=slots.cuda(), rotary=rot, left_out=left)
        assert int(left) == 2
        check_states(state, want)
    Lq = L + 3
    H = heads * group
    Q = rows(gen, dt, B, H, Lq, d, packed=True)
    rot = make_rot(fs, kind, d, B, Lq, gen)
    read = torch.tensor([5, 5, 7, 1, 99, 0], dtype=torch.int32)           # 1 is empty, 99 no slot
    lengths = torch.tensor([Lq, 2, Lq, 1, 3, 0], dtype=torch.int32)
    q = turned(Q.double().cpu(), rot)
    ref = torch.zeros((B, H, Lq, dv), dtype=torch.float64)
    for b in range(B):
        m = int(lengths[b])
        Q[b, :, m:] = float("nan")
        if b in (3, 4):
            continue
        for h in range(H):
            ref[b, h, :m] = o.read(want[int(read[b])][h // group], h // group, q[b, h, :m])
    unread = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = fs.state_attention(f, state, Q, lengths=lengths.cuda(), slots=read.cuda(), rotary=rot, out=empty_rows(dt, B, H, Lq, dv), unread=unread)
    check(Y, ref, F32, "Y")
    assert int(unread) == 4 * H
    check(fs.state_attention(f, state, Q, lengths=lengths.cuda(), slots=read.cuda(), rotary=rot,
                             out=empty_rows(torch.float32, B, H, Lq, dv)), ref, F32, "Y in fp32")


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:7]))
def test_backward(fs, shape):
    """Gradients of queries, states, keys and values against the formulas; slots shared by sequences, slots that nobody reads, padding."""
    import torch
    d, dv, M, heads, group, L, dtype, family, kind = shape
    B, nslots = 4, 5
    gen, o, f, dt = setup(fs, shape, B, 31 + d)
    H = heads * group
    K, V = rows(gen, dt, B, heads, L, d), rows(gen, dt, B, heads, L, dv, packed=True)
    klen = torch.tensor([L, max(1, L // 2), 0, L], dtype=torch.int32)
    slots = torch.tensor([4, 1, 0, 2], dtype=torch.int32)
    rk = make_rot(fs, kind, d, B, L, gen)
    k, v = turned(K.double().cpu(), rk), V.double().cpu()
    state = fs.state_new(nslots, heads, M, dv)
    want = oracle_states(o, B, nslots, dv)
    for b in range(B):
        for h in range(heads):
            n = int(klen[b])
            want[int(slots[b])][h] = o.append(want[int(slots[b])][h], b, h, k[b, h, :n], v[b, h, :n])
        K[b, :, n:], V[b, :, n:] = float("nan"), float("nan")
    fs.state_append(f, state, K, V, lengths=klen.cuda(), slots=slots.cuda(), rotary=rk)
    Lq = L + 2
    Q, dY = rows(gen, dt, B, H, Lq, d), rows(gen, dt, B, H, Lq, dv, packed=True)
    qlen = torch.tensor([Lq, 1, Lq, max(1, Lq - 5)], dtype=torch.int32)
    read = torch.tensor([4, 1, 0, 4], dtype=torch.int32)            # 0 and 3 share a state; 0 is empty
    rq = make_rot(fs, kind, d, B, Lq, gen)
    q, dy = turned(Q.double().cpu(), rq), dY.double().cpu()
    rdq = torch.zeros_like(q)
    rT, rz = torch.zeros((nslots, heads, M, dv), dtype=torch.float64), torch.zeros((nslots, heads, M), dtype=torch.float64)
    for b in range(B):
        n = int(qlen[b])
        for h in range(H):
            dq, dT, dz = o.read_backward(want[int(read[b])][h // group], h // group, q[b, h, :n], dy[b, h, :n])
            rdq[b, h, :n] = dq
            rT[read[b], h // group] += dT
            rz[read[b], h // group] += dz
        Q[b, :, n:], dY[b, :, n:] = float("nan"), float("nan")
    rdq = turned(rdq, rq, True)
    dQ, ds = fs.state_attention_backward(f, state, Q, dY, lengths=qlen.cuda(), slots=read.cuda(), rotary=rq, dQ=empty_rows(dt, B, H, Lq, d))
    # (with one feature, or one key, the true gradient of the queries is zero: its rounding is measured against what is subtracted)
    floor = float(dy.norm()) * max(1.0, float(v[v.isfinite()].abs().max())) * 1e-6 * (1 + d)
    if float(rdq.norm()) <= 100 * floor:
        off = float((dQ.double().cpu() - rdq).norm())
        assert off <= floor + (HALF + GRAD) * float(rdq.norm()), (off, floor)
    else:
        mean = max(float((T.norm(dim=1) / z.clamp_min(1e-300)).max()) for row in want for T, z, _ in row)
        size = 1.1 * dy.norm(dim=-1, keepdim=True) * mean * float(o.s * o.W1.norm(dim=-1).max())
        check(dQ, rdq, GRAD, "dQ", size.nan_to_num(0.0) / 50)         # 10 GRAD / 50 = 2e-5
    check(ds.T.reshape(1, -1), rT.reshape(1, -1), F32, "dT")
    check(ds.z.reshape(1, -1), rz.reshape(1, -1), GRAD, "dz")
    assert bool((ds.T[3] == 0).all()) and bool((ds.z[3] == 0).all())
    # keys and values, from a gradient of the state of any size
    gT, gz = torch.randn((nslots, heads, M, dv), generator=gen), torch.randn((nslots, heads, M), generator=gen)
    dK, dV = fs.state_append_backward(f, state, fs.State(gT.cuda(), gz.cuda(), None), K, V, lengths=klen.cuda(), slots=slots.cuda(), rotary=rk,
                                      grads=(empty_rows(dt, B, heads, L, d), empty_rows(dt, B, heads, L, dv)))
    rdk, rdv = torch.zeros_like(k), torch.zeros_like(v)
    for b in range(B):
        n, s = int(klen[b]), int(slots[b])
        for h in range(heads):
            if n:
                rdk[b, h, :n], rdv[b, h, :n] = o.append_backward(want[s][h][2], h, k[b, h, :n], v[b, h, :n], gT[s, h].double(), gz[s, h].double())
    check(dK, turned(rdk, rk, True), GRAD, "dK")
    check(dV, rdv, F32, "dV")


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:7]))
def test_step(fs, shape):
    """Single tokens: onto states with keys and onto empty ones, a sequence without a slot, one whose slot is taken."""
    import torch
    d, dv, M, heads, group, L, dtype, family, kind = shape
    B, nslots, H = 5, 6, heads * group
    gen, o, f, dt = setup(fs, shape, B, 47 + d)
    state, want = fs.state_new(nslots, heads, M, dv), oracle_states(o, B, nslots, dv)
    state.T.fill_(float("nan"))                     # (an empty state's T and z are not read)
    slots = torch.tensor([3, 3, 6, 1, 0], dtype=torch.int32)
    for turn in range(3):
        Q, K, V = (rows(gen, dt, B, n, 1, c, 1.0 + 0.5 * turn, packed=True) for n, c in ((H, d), (heads, d), (heads, dv)))
        rot = make_rot(fs, kind, d, B, 1, gen)
        q, k, v = turned(Q.double().cpu(), rot), turned(K.double().cpu(), rot), V.double().cpu()
        ref = torch.zeros((B, H, 1, dv), dtype=torch.float64)
        for b in (0, 3, 4):
            for h in range(heads):
                want[int(slots[b])][h] = o.append(want[int(slots[b])][h], b, h, k[b, h], v[b, h])
            for h in range(H):
                ref[b, h] = o.read(want[int(slots[b])][h // group], h // group, q[b, h])
        unread = torch.zeros(1, dtype=torch.int32, device="cuda")
        Y = fs.state_step(f, state, Q, K, V, slots=slots.cuda(), rotary=rot, out=empty_rows(dt, B, H, 1, dv), unread=unread)
        check(Y, ref, F32, ("Y", turn))
        assert int(unread) == 2 * H
    live = fs.State(*(t[[3, 1, 0]] for t in state))
    check_states(live, [want[3], want[1], want[0]])
    assert bool(torch.isnan(state.T[2]).all()) and float(state.shift[2, 0]) == -math.inf       # nobody's slot stays as it was


def test_gradients_against_differences(fs):
    """The oracle's gradients, which the kernels are held to above, against central differences of its own forward pass (in 64 bits)."""
    import torch
    gen = torch.Generator().manual_seed(3)
    d, dv, M, n, nq = 6, 5, 12, 7, 4
    o = Oracle(make_theta(gen, "dense", 1, d), torch.randn((1, M, d), generator=gen), d ** -0.25, 1)
    k, v, q, dy = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((n, d), (n, dv), (nq, d), (nq, dv)))
    def loss(k, v, q):
        st = oracle_states(o, 1, 1, dv)[0][0]
        return (o.read(o.append(st, 0, 0, k, v), 0, q) * dy).sum()
    st = o.append(oracle_states(o, 1, 1, dv)[0][0], 0, 0, k, v)
    dq, dT, dz = o.read_backward(st, 0, q, dy)
    dk, dvv = o.append_backward(st[2], 0, k, v, dT, dz)
    for x, g, i in ((k, dk, 0), (v, dvv, 1), (q, dq, 2)):
        for r in range(x.shape[0]):
            for c in range(x.shape[1]):
                a = [k, v, q]
                up, down = x.clone(), x.clone()
                up[r, c] += 1e-5
                down[r, c] -= 1e-5
                diff = (loss(*(a[:i] + [up] + a[i + 1:])) - loss(*(a[:i] + [down] + a[i + 1:]))) / 2e-5
                assert abs(float(diff - g[r, c])) <= 1e-7 * (1 + abs(float(g[r, c])))


# ------------------------------------------------------------------------------------------------ together, and with the rest of the library
def test_prompt_and_tokens_are_causal_attention(fs):
    """A prompt appended, then tokens one by one: rows of favorsharp_attention(causal) of the whole sequence (1e-4: its bar in fp32)."""
    import torch
    gen = torch.Generator().manual_seed(5)
    B, H, L, L0, d, M = 2, 3, 50, 37, 64, 256
    s = d ** -0.25
    Q, K, V = (rows(gen, torch.float32, B, H, L, d) for _ in range(3))
    theta, omega = fs.fit_params("sderf", Q, K, s, groups=H), torch.randn((H, M, d), generator=gen).cuda()
    Y = fs.attention(theta, Q, K, V, s, omega, causal=True)
    f, state = fs.state_prepare(theta, omega, s), fs.state_new(B, H, M, d)
    fs.state_append(f, state, K[:, :, :L0], V[:, :, :L0], fresh=True)
    for t in range(L0, L):
        y = fs.state_step(f, state, Q[:, :, t:t + 1], K[:, :, t:t + 1], V[:, :, t:t + 1])
        check(y, Y[:, :, t:t + 1].double().cpu(), 1e-4, t)


@pytest.mark.parametrize("variant", ["sderf", "aderf"])
def test_cross_attention_of_a_padded_batch_is_attention_of_each(fs, variant):
    """Forward and backward through states against favorsharp_attention on each sequence's own keys (general fp32 kernels)."""
    import torch
    gen = torch.Generator().manual_seed(6)
    B, H, Lq, Lk, d, M = 3, 2, 45, 70, 32, 96
    s = d ** -0.25
    Q, K, V, dY = (rows(gen, torch.float32, B, H, n, d) for n in (Lq, Lk, Lk, Lq))
    theta, omega = fs.fit_params(variant, K, K, s, groups=H), torch.randn((H, M, d), generator=gen).cuda()
    n = torch.tensor([70, 1, 33], dtype=torch.int32, device="cuda")
    f, state = fs.state_prepare(theta, omega, s), fs.state_new(B, H, M, d)
    fs.state_append(f, state, K, V, lengths=n, fresh=True)
    Y = fs.state_attention(f, state, Q)
    dQ, ds = fs.state_attention_backward(f, state, Q, dY)
    dK, dV = fs.state_append_backward(f, state, ds, K, V, lengths=n)
    for b in range(B):
        m = int(n[b])
        one = [t[b:b + 1] for t in (Q, K[:, :, :m], V[:, :, :m], dY)]
        check(Y[b:b + 1], fs.attention(theta, *one[:3], s, omega).double().cpu(), 1e-4, "Y")
        g = fs.attention_backward(theta, *one, s, omega)
        scale = float(dY.norm() * V.abs().max())
        for got, ref in zip((dQ[b:b + 1], dK[b:b + 1, :, :m], dV[b:b + 1, :, :m]), g):
            assert float((got - ref).norm()) <= 3e-4 * float(ref.norm()) + 1e-6 * scale
        assert bool((dK[b, :, m:] == 0).all()) and bool((dV[b, :, m:] == 0).all())


def test_many_sequences_and_long_ones(fs):
    """More workgroups than a pass of the chip, splits of long rows and their join, against the same in float64 on the GPU."""
    import torch
    for B, H, G, L, d, M, dt in ((40, 4, 1, 33, 64, 256, torch.bfloat16), (1, 2, 2, 5000, 64, 256, torch.float32), (2, 1, 1, 3001, 128, 512, torch.bfloat16)):
        gen = torch.Generator().manual_seed(L)
        s = d ** -0.25
        theta, omega = make_theta(gen, "iso", 1, d).cuda(), torch.randn((1, M, d), generator=gen).cuda()
        K, V, Q = (rows(gen, dt, B, h, L, d) for h in (H, H, H * G))
        f, state = fs.state_prepare(theta, omega, s, heads=H), fs.state_new(B, H, M, d)
        fs.state_append(f, state, K, V, fresh=True)
        Y = fs.state_attention(f, state, Q)
        o = Oracle(theta.cpu(), omega.cpu(), s, 1)
        W1, W2, bias = (t[0].cuda() for t in (o.W1, o.W2, o.bias))
        k = s * K.double()
        e = k @ W2.T + bias - 0.5 * (k * k).sum(-1, keepdim=True)
        top = e.amax((2, 3), keepdim=True)
        S = torch.exp(e - top)
        T, z = S.transpose(2, 3) @ V.double(), S.sum(2)
        check(state.T.flatten(2), T.flatten(2).cpu(), F32, "T")
        check(state.z, z.cpu(), F32, "z")
        e = (s * Q.double()).reshape(B, H, -1, d) @ W1.T + bias
        P = torch.exp(e - e.amax(-1, keepdim=True))
        check(Y.reshape(B, H, -1, d), ((P @ T) / (P @ z[..., None])).cpu(), F32, "Y")


def test_results_do_not_change_from_run_to_run(fs):
    import torch
    shape = SHAPES[0]
    gen, o, f, dt = setup(fs, shape, 3, 1)
    d, dv, M, heads = shape[:4]
    K, V, Q, dY = (rows(gen, dt, 3, heads, 300, d) for _ in range(4))
    def all_of():
        state = fs.state_new(3, heads, M, dv)
        fs.state_append(f, state, K, V)
        fs.state_append(f, state, K, V)
        dQ, ds = fs.state_attention_backward(f, state, Q, dY)
        out = [fs.state_attention(f, state, Q), dQ, ds.T, ds.z, *fs.state_append_backward(f, state, ds, K, V)]
        out.append(fs.state_step(f, state, Q[:, :, :1], K[:, :, :1], V[:, :, :1]))
        return out + list(state)
    a, b = all_of(), all_of()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_and_on_other_streams(fs):
    """A step and a padded append with its backward, captured on a stream of their own and replayed on new data, with eager calls between."""
    import torch
    gen, o, f, dt = setup(fs, SHAPES[1], 2, 9)
    d, dv, M, heads, group = SHAPES[1][:5]
    B, L, H = 2, 50, heads * group
    K, V = rows(gen, dt, B, heads, L, d), rows(gen, dt, B, heads, L, dv)
    Q, q1, k1, v1 = (rows(gen, dt, B, *n) for n in ((H, L, d), (H, 1, d), (heads, 1, d), (heads, 1, dv)))
    n = torch.tensor([50, 20], dtype=torch.int32, device="cuda")
    rot = make_rot(fs, ("half", 1.0), d, B, L, gen)
    one = make_rot(fs, ("half", 1.0), d, B, 1, gen)
    state = fs.state_new(B, heads, M, dv)
    def work():
        fs.state_append(f, state, K, V, lengths=n, rotary=rot, fresh=True)
        dQ, ds = fs.state_attention_backward(f, state, Q, Q if dv == d else Q[..., :dv], rotary=rot)
        dK, dV = fs.state_append_backward(f, state, ds, K, V, lengths=n, rotary=rot)
        return [fs.state_step(f, state, q1, k1, v1, rotary=one), dQ, dK, dV, fs.rotary(Q, rot), *state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for i in range(3):
        for t in (K, V, Q, q1, k1, v1):
            t.copy_(torch.randn(t.shape, generator=gen).to(dt))
        n.copy_(torch.tensor([50 - i, 1 + i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_refusals_on_the_device(fs):
    import torch
    gen, o, f, dt = setup(fs, SHAPES[0], 2, 2)
    d, dv, M, heads = SHAPES[0][:4]
    K, V, Q = (rows(gen, dt, 2, heads, 8, d) for _ in range(3))
    state = fs.state_new(2, heads, M, dv)
    before = [t.clone() for t in state]
    for call in (lambda: fs.state_append(f, state, K, V.float()),                                          # two dtypes
                 lambda: fs.state_append(f, state, K, V, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")),
                 lambda: fs.state_append(f, state, K[..., :60], V),
                 lambda: fs.state_append(f, state, K[:, :1], V[:, :1]),
                 lambda: fs.state_append(f, state, K, V, lengths=torch.tensor([1, 2], device="cuda")),     # 64-bit lengths
                 lambda: fs.state_append(f, state, K, V, slots=torch.tensor([1], dtype=torch.int32, device="cuda")),
                 lambda: fs.state_append(f, fs.state_new(1, heads, M, dv), K, V),
                 lambda: fs.state_attention(f, fs.state_new(2, heads, M + 1, dv), Q),
                 lambda: fs.state_attention(f, state, Q.transpose(2, 3)),
                 lambda: fs.state_step(f, state, Q, K, V),
                 lambda: fs.rotary(Q, fs.Rotary(fs.rotary_frequencies(66), None)),
                 lambda: fs.rotary(Q, fs.Rotary(fs.rotary_frequencies(64).float(), None)),
                 lambda: fs.rotary(Q, fs.Rotary(fs.rotary_frequencies(64, device="cpu"), None)),
                 lambda: fs.rotary(Q, fs.Rotary(fs.rotary_frequencies(64), None), out=Q[:, :, :, :].transpose(0, 1).contiguous().transpose(0, 1)[:, :1])):
        with pytest.raises((ValueError, fs.FavorSharpError)):
            call()
    assert all(torch.equal(a, b) for a, b in zip(before, state))
