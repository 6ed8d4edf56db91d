"""Linear attention with a decay for each head against the recurrence in 64 bits, through the public entry points.

Tolerances, relative to the norm of a result.  fp32: a power of lambda, its product, a score and its product with a row are each off by
at most one half step (2^-24) of themselves, twice that where a state is decayed, and a sum of n products of random sign by sqrt(n) half steps of its
norm, n <= 128 numbers of a row + 64 rows of a chunk; the chunks' sums by one each, of at most 32 here: 8 + 14 + 6 < 32 half steps of 2^-24 =
2e-6.  Gradients have one product more and sums over four query heads: F32 = 4e-6 for all.  bf16 results: half a step, 2^-8 of each number,
and scores, states and their products to 16 bits, 3 * 2^-17 < 2^-15: BF16 = 2^-8 + 2^-15.  (In the norm a rounding is 2^-8 only if every number
is at its worst.)  Numbers of a result can be far smaller than the result: single ones are held to its largest times the tolerance.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

F32 = 4e-6
BF16 = 2.0 ** -8 + 2.0 ** -15


@pytest.fixture(scope="module")
def fs():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2302_00787_amd import binding
    binding.lib()
    return binding


# ------------------------------------------------------------------------------------------------ the recurrence in 64 bits
def forward(q, k, v, g, s, S0, n):
    """q [H,L,d], k [Hk,L,d], v [Hk,L,dv] of one sequence of n rows -> Y, S."""
    import torch
    H, L, d = q.shape
    Hk, G = k.shape[0], H // k.shape[0]
    lam = torch.exp(torch.clamp(g, max=0.0))[:, None, None]
    S, Y = S0.clone(), torch.zeros(H, L, v.shape[2], dtype=torch.float64)
    for i in range(n):
        S = lam * S + k[:, i, :, None] * v[:, i, None, :]
        Y[:, i] = s * (q[:, i].reshape(Hk, G, d) @ S).reshape(H, -1)
    return Y, S


def backward(q, k, v, dy, g, s, S0, dS, n):
    import torch
    H, L, d = q.shape
    Hk, G = k.shape[0], H // k.shape[0]
    lam = torch.exp(torch.clamp(g, max=0.0))[:, None, None]
    dq, dk, dv = (torch.zeros_like(t) for t in (q, k, v))
    S, states = S0.clone(), []
    for i in range(n):
        S = lam * S + k[:, i, :, None] * v[:, i, None, :]
        states.append(S)
    D = dS.clone()
    for i in reversed(range(n)):
        y = dy[:, i].reshape(Hk, G, -1)
        dq[:, i] = s * (y @ states[i].transpose(1, 2)).reshape(H, d)
        D = D + s * q[:, i].reshape(Hk, G, d).transpose(1, 2) @ y
        dk[:, i] = (D @ v[:, i, :, None])[..., 0]
        dv[:, i] = (D.transpose(1, 2) @ k[:, i, :, None])[..., 0]
        D = lam * D
    return dq, dk, dv, D


def close(got, want, tol):
    got, want = got.detach().double().cpu(), want.double()
    assert got.isfinite().all()
    off = (got - want)
    assert off.norm() <= tol * want.norm() + 1e-30, (float(off.norm()), float(want.norm()))
    if want.numel():
        assert off.abs().max() <= 4 * tol * want.abs().max() + 1e-30


def tolerance(dtype):
    return F32 if dtype == "f32" else BF16


def dtype_of(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def rows(fs, gen, dtype, *shape, pad=0.0):
    """A tensor whose rows start at multiples of 16 bytes, whatever its width; what lies behind its rows is `pad`."""
    import torch
    wide = torch.full((*shape[:-1], (shape[-1] + 7) // 8 * 8 + 8), pad, dtype=dtype_of(dtype))
    t = wide[..., :shape[-1]]
    t.copy_(torch.randn(shape, generator=gen))
    return wide.cuda()[..., :shape[-1]]


def decays(kind, heads):
    import torch
    return {"none": torch.zeros(heads), "slow": -2.0 ** -(5.0 + torch.arange(heads)), "steep": -2.0 ** -torch.arange(heads).float(),
            "mixed": torch.tensor([0.0, -0.01, -3.0, -math.inf] * heads)[:heads], "huge": torch.full((heads,), -200.0)}[kind].contiguous()


class Case:
    def __init__(self, fs, dtype, B, H, Hk, L, d, dv, decay, lengths=None, pad=0.0, seed=0):
        import torch
        gen = torch.Generator().manual_seed(1000 * L + 10 * d + dv + seed)
        self.fs, self.dtype, self.B, self.H, self.Hk, self.L, self.d, self.dv = fs, dtype, B, H, Hk, L, d, dv
        self.Q, self.K, self.V, self.dY = (rows(fs, gen, dtype, B, h, L, w, pad=pad) for h, w in ((H, d), (Hk, d), (Hk, dv), (H, dv)))
        self.n = [L] * B if lengths is None else lengths
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
        for b, m in enumerate(self.n):          # what padding holds does not matter
            for t in (self.Q, self.K, self.V, self.dY):
                t[b, :, max(m, 0):] = math.nan
        self.g, self.s = decays(decay, Hk).cuda(), 0.7
        self.S0 = torch.randn((B, Hk, d, dv), generator=gen).cuda()
        self.dS = torch.randn((B, Hk, d, dv), generator=gen).cuda()

    def host(self, b):
        import torch
        m = max(0, min(self.n[b], self.L))
        out = []
        for t in (self.Q, self.K, self.V, self.dY):
            x = t[b].detach().double().cpu()
            x[:, m:] = 0.0
            out.append(x)
        return (*out, self.g.double().cpu(), m)

    def forward(self, b, S0=None):
        import torch
        q, k, v, _, g, m = self.host(b)
        return forward(q, k, v, g, self.s, torch.zeros(self.Hk, self.d, self.dv, dtype=torch.float64) if S0 is None else S0.double().cpu(), m)

    def backward(self, b, S0=None, dS=None):
        import torch
        q, k, v, dy, g, m = self.host(b)
        zero = torch.zeros(self.Hk, self.d, self.dv, dtype=torch.float64)
        return backward(q, k, v, dy, g, self.s, zero if S0 is None else S0.double().cpu(), zero if dS is None else dS.double().cpu(), m)


SIZES = [            # B, H, Hk, L, d, dv
    (1, 1, 1, 1, 8, 8), (2, 2, 2, 2, 16, 16), (1, 2, 1, 63, 32, 32), (2, 4, 2, 64, 64, 64), (1, 3, 1, 65, 24, 40), (2, 2, 2, 130, 128, 128),
    (1, 4, 1, 77, 96, 128), (1, 2, 2, 200, 16, 128), (1, 2, 2, 129, 128, 16), (1, 8, 2, 190, 64, 32), (1, 1, 1, 5, 1, 1), (2, 2, 1, 70, 3, 5),
    (1, 2, 2, 66, 33, 65), (1, 2, 1, 100, 127, 31),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("states", [False, True])
def test_rows_and_gradients(fs, dtype, size, states):
    import torch
    c = Case(fs, dtype, *size, decay="mixed" if states else "slow", pad=math.nan)
    before, after = (c.S0, torch.full_like(c.S0, math.nan)) if states else (None, None)
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=before, after=after)
    got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=before, dafter=c.dS if states else None)
    assert got[3] is None or states
    for b in range(c.B):
        y, S = c.forward(b, c.S0[b] if states else None)
        close(Y[b], y, tolerance(dtype))
        if states:
            close(after[b], S, F32)
        want = c.backward(b, c.S0[b] if states else None, c.dS[b] if states else None)
        for x, w in zip(got[:3], want):
            close(x[b], w, tolerance(dtype))
        if states:
            close(got[3][b], want[3], F32)


@pytest.mark.parametrize("dtype,B,H,Hk,L,d,dv", [("bf16", 1, 2, 2, 1000, 64, 64), ("f32", 1, 2, 1, 777, 48, 64), ("bf16", 2, 4, 2, 643, 128, 96),
                                                 ("f32", 2, 1, 1, 1025, 128, 128), ("bf16", 1, 1, 1, 2000, 20, 30)])
@pytest.mark.parametrize("decay", ["none", "mixed", "steep"])
def test_segments(fs, dtype, B, H, Hk, L, d, dv, decay):
    """Long sequences of few states are shared out, also those of a padded batch that end in any segment."""
    import torch
    for lengths in (None, [L, L // 3][:B], [0, L - 1][:B]):
        c = Case(fs, dtype, B, H, Hk, L, d, dv, decay, lengths)
        after = torch.empty_like(c.S0)
        Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=c.S0, after=after, lengths=c.lengths)
        got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=c.S0, dafter=c.dS, lengths=c.lengths)
        for b in range(B):
            y, S = c.forward(b, c.S0[b])
            close(Y[b], y, tolerance(dtype))
            close(after[b], S, F32)
            want = c.backward(b, c.S0[b], c.dS[b])
            for x, w in zip(got[:3], want):
                close(x[b], w, tolerance(dtype))
            close(got[3][b], want[3], F32)


def test_segments_in_place(fs):
    """States before and after in one pool, sequences long enough to be shared out."""
    import torch
    c = Case(fs, "f32", 2, 2, 1, 700, 32, 32, "slow", [700, 500])
    pool = c.S0.clone()
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=pool, after=pool, lengths=c.lengths)
    for b in range(2):
        y, S = c.forward(b, c.S0[b])
        close(Y[b], y, F32)
        close(pool[b], S, F32)


@pytest.mark.parametrize("lengths", [[0, 1, 63, 64], [65, 100, -3, 1000], [128, 127, 0, 0]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_padded_batches(fs, dtype, lengths):
    import torch
    c = Case(fs, dtype, 4, 4, 2, 128, 64, 64, "mixed", lengths)
    pool = c.S0.clone()
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=pool, after=pool, lengths=c.lengths)
    got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=c.S0, dafter=c.dS, lengths=c.lengths)
    for b, n in enumerate(lengths):
        m = max(0, min(n, c.L))
        y, S = c.forward(b, c.S0[b])
        close(Y[b], y, tolerance(dtype))
        assert (Y[b, :, m:] == 0).all() and all((t[b, :, m:] == 0).all() for t in got[:3])
        close(pool[b], S, F32)
        if m == 0:
            assert torch.equal(pool[b], c.S0[b]) and torch.equal(got[3][b], c.dS[b])
        want = c.backward(b, c.S0[b], c.dS[b])
        for x, w in zip(got[:3], want):
            close(x[b], w, tolerance(dtype))
        close(got[3][b], want[3], F32)


def test_gradients_of_several_dtypes_and_more_slots_than_sequences(fs):
    """dQ in fp32, dK and dV in bf16; a pool with slots that no sequence has: zeros there."""
    import torch
    for d in (64, 96):
        c = Case(fs, "bf16", 2, 4, 2, 90, d, d, "slow")
        start = torch.randn((5, 2, d, d), generator=torch.Generator().manual_seed(5)).cuda()
        grads = [torch.empty(t.shape, dtype=dt, device="cuda") for t, dt in ((c.Q, torch.float32), (c.K, torch.bfloat16), (c.V, torch.bfloat16))]
        got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=start, grads=grads)
        assert all(x is y for x, y in zip(got, grads)) and (got[3][2:] == 0).all()
        for b in range(2):
            want = c.backward(b, start[b])
            for x, w, tol in zip(got, want, (F32, BF16, BF16, F32)):
                close(x[b], w, tol)


@pytest.mark.parametrize("L,H,Hk", [(1, 4, 2), (64, 6, 2), (700, 4, 1)])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 128), ("bf16", 128)])
def test_heads_that_share_states(fs, dtype, d, L, H, Hk):
    """Few states: every query head has a workgroup of its own; many: they go together.  Sequences that are left out among them."""
    import torch
    for B, check in ((3, (0, 2)), (260, (0, 131, 259))):
        if B * L > 20000:
            continue
        c = Case(fs, dtype, B, H, Hk, L, d, 64, "slow")
        slots = torch.arange(B, dtype=torch.int32).cuda()
        slots[1] = 0
        pool = c.S0.clone()
        Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=pool, after=pool, slots=slots)
        got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=c.S0, dafter=c.dS, slots=slots)
        assert (Y[1] == 0).all() and all((x[1] == 0).all() for x in got[:3])
        assert torch.equal(pool[1], c.S0[1]) and (got[3][1] == 0).all()
        for b in check:
            y, S = c.forward(b, c.S0[b])
            close(Y[b], y, tolerance(dtype))
            close(pool[b], S, F32)
            want = c.backward(b, c.S0[b], c.dS[b])
            for x, w in zip(got[:3], want):
                close(x[b], w, tolerance(dtype))
            close(got[3][b], want[3], F32)


@pytest.mark.parametrize("dtype,L", [("bf16", 130), ("f32", 33)])
def test_many_heads_of_one_state(fs, dtype, L):
    import torch
    c = Case(fs, dtype, 1, 64, 1, L, 64, 64, "slow")
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s)
    got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s)
    close(Y[0], c.forward(0)[0], tolerance(dtype))
    for x, w in zip(got[:3], c.backward(0)):
        close(x[0], w, tolerance(dtype))
    pool = torch.zeros((1, 1, 64, 64), device="cuda")
    for i in range(3):
        y = fs.decay_step(pool, *(x[:, :, i:i + 1] for x in (c.Q, c.K, c.V)), c.g, c.s)
        close(y[0, :, 0], c.forward(0)[0][:, i], tolerance(dtype))


def test_one_row_of_any_stride(fs):
    """Sequences of one row: from row to row their tensors may have any stride."""
    import torch
    c = Case(fs, "bf16", 2, 2, 2, 1, 64, 64, "slow")
    far = [torch.as_strided(t.contiguous(), t.shape, (128, 64, 1 << 33, 1)) for t in (c.Q, c.K, c.V, c.dY)]
    Y = fs.decay_attention(*far[:3], c.g, c.s, before=c.S0)
    assert torch.equal(Y, fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=c.S0))
    got, want = (fs.decay_attention_backward(*t, c.g, c.s, before=c.S0) for t in (far, (c.Q, c.K, c.V, c.dY)))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert torch.equal(fs.decay_step(c.S0.clone(), *far[:3], c.g, c.s), fs.decay_step(c.S0.clone(), c.Q, c.K, c.V, c.g, c.s))


def test_no_rows(fs):
    import torch
    c = Case(fs, "bf16", 2, 2, 2, 0, 64, 64, "slow")
    after = torch.full_like(c.S0, math.nan)
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=c.S0, after=after)
    assert Y.numel() == 0 and torch.equal(after, c.S0)
    fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, after=after)
    assert (after == 0).all()
    got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=c.S0, dafter=c.dS)
    assert torch.equal(got[3], c.dS)


def test_results_of_the_other_dtype(fs):
    """bf16 rows, results in fp32: their accuracy; fp32 rows, results in bf16."""
    import torch
    c = Case(fs, "bf16", 1, 2, 1, 300, 64, 96, "slow")
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=c.S0, out_dtype=torch.float32)
    close(Y[0], c.forward(0, c.S0[0])[0], F32)
    for x, w in zip(fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, grad_dtype=torch.float32), c.backward(0)):
        if x is not None:
            close(x[0], w, F32)
    c = Case(fs, "f32", 1, 2, 1, 300, 64, 96, "slow")
    close(fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, out_dtype=torch.bfloat16)[0], c.forward(0)[0], BF16)


def test_powers_of_long_sequences(fs):
    """lambda near one over many rows: no error of a factor is repeated.  Ones as keys and values: S is the sum of the powers."""
    import torch
    L = 65536
    K = torch.ones((1, 3, L, 8), device="cuda")
    g = torch.tensor([0.0, -2.0 ** -17, -2.0 ** -12], device="cuda")
    after = fs.decay_state_new(1, 3, 8, 8)
    Y = fs.decay_attention(K, K, K, g, 0.125, after=after)
    n = torch.arange(1, L + 1, dtype=torch.float64)
    want = torch.stack([n, torch.expm1(n * g[1].item()) / math.expm1(g[1].item()), torch.expm1(n * g[2].item()) / math.expm1(g[2].item())])
    # sums of up to 1024 chunks of positive numbers: a half step of the sum at each, at random: 32 * 2^-24
    assert ((Y[0, :, :, 0].double().cpu() - want).abs() / want).max() <= 2 * 32 * 2.0 ** -24
    assert ((after[0, :, 0, 0].double().cpu() - want[:, -1]).abs() / want[:, -1]).max() <= 2 * 32 * 2.0 ** -24


@pytest.mark.parametrize("decay", ["huge", "mixed"])
def test_a_state_that_is_all_there_is(fs, decay):
    """Large states before rows of zeros: what is left of them, to their own accuracy."""
    import torch
    c = Case(fs, "f32", 1, 4, 4, 70, 32, 32, decay)
    c.K.zero_()
    S0 = 1e6 * c.S0
    after = torch.empty_like(S0)
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=S0, after=after)
    y, S = c.forward(0, S0[0])
    for h in range(4):
        for r in range(70):
            w = y[h, r]
            assert (Y[0, h, r].double().cpu() - w).norm() <= F32 * w.norm() + 1e-35
        close(after[0, h], S[h], F32)


# ------------------------------------------------------------------------------------------------ tokens
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,Hk,d,dv", [(1, 1, 1, 1, 1), (3, 4, 2, 64, 64), (2, 6, 2, 24, 40), (5, 8, 2, 128, 128), (2, 2, 2, 17, 33), (300, 2, 2, 64, 64),
                                         (257, 4, 2, 96, 50), (130, 16, 4, 128, 36)])
def test_tokens(fs, dtype, B, H, Hk, d, dv):
    import torch
    c = Case(fs, dtype, B, H, Hk, 3, d, dv, "mixed")
    pool = c.S0.clone()
    ys = [fs.decay_step(pool, c.Q[:, :, i:i + 1], c.K[:, :, i:i + 1], c.V[:, :, i:i + 1], c.g, c.s) for i in range(3)]
    for b in (range(B) if B < 9 else [0, B // 2, B - 1]):
        y, S = c.forward(b, c.S0[b])
        close(torch.cat(ys, 2)[b], y, tolerance(dtype))
        close(pool[b], S, F32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_go_on_where_prompts_end(fs, dtype):
    """A prompt in one call, in two, or token by token; slots in any order, those that no sequence names as they were."""
    import torch
    c = Case(fs, dtype, 2, 4, 2, 131, 64, 64, "slow")
    slots = torch.tensor([3, 1], dtype=torch.int32).cuda()
    start = torch.randn((5, 2, 64, 64), generator=torch.Generator().manual_seed(1)).cuda()
    cuts = ([0, 131], [0, 67, 131], [0, 128, 131], [0, 130, 131])
    for cut in cuts:
        pool = start.clone()
        Y = [fs.decay_attention(*(t[:, :, a:z] for t in (c.Q, c.K, c.V)), c.g, c.s, before=pool, after=pool, slots=slots)
             if z - a > 1 else fs.decay_step(pool, *(t[:, :, a:z] for t in (c.Q, c.K, c.V)), c.g, c.s, slots=slots) for a, z in zip(cut, cut[1:])]
        for b, at in enumerate((3, 1)):
            y, S = c.forward(b, start[at])
            close(torch.cat(Y, 2)[b], y, tolerance(dtype))
            close(pool[at], S, F32)
        for at in (0, 2, 4):
            assert torch.equal(pool[at], start[at])


# ------------------------------------------------------------------------------------------------ slots
def test_sequences_that_are_left_out(fs):
    """Slots outside the pool, and the same one twice, where states are written: zeros, the states as they were, counted."""
    import torch
    c = Case(fs, "f32", 5, 2, 2, 70, 32, 32, "slow")
    slots = torch.tensor([2, 7, 2, -1, 0], dtype=torch.int32).cuda()
    start = torch.randn((4, 2, 32, 32), generator=torch.Generator().manual_seed(2)).cuda()
    for step in (False, True):
        pool, count = start.clone(), torch.tensor([10], dtype=torch.int32).cuda()
        r = slice(0, 1) if step else slice(0, 70)
        t = [x[:, :, r] for x in (c.Q, c.K, c.V)]
        Y = fs.decay_step(pool, *t, c.g, c.s, slots=slots, left_out=count) if step else \
            fs.decay_attention(*t, c.g, c.s, before=pool, after=pool, slots=slots, left_out=count)
        assert count.item() == 13
        for b, at in ((0, 2), (4, 0)):
            q, k, v, _, g, m = c.host(b)
            y, S = forward(q[:, r], k[:, r], v[:, r], g, c.s, start[at].double().cpu(), r.stop)
            close(Y[b], y, F32)
            close(pool[at], S, F32)
        for b in (1, 2, 3):
            assert (Y[b] == 0).all()
        assert torch.equal(pool[1], start[1]) and torch.equal(pool[3], start[3])
    got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=start, dafter=start, slots=slots)
    for b, at in ((0, 2), (4, 0)):
        want = c.backward(b, start[at], start[at])
        for x, w in zip(got[:3], want):
            close(x[b], w, F32)
        close(got[3][at], want[3], F32)
    for b in (1, 2, 3):
        assert all((x[b] == 0).all() for x in got[:3])
    assert (got[3][1] == 0).all() and (got[3][3] == 0).all()


@pytest.mark.parametrize("L", [70, 600])
def test_sequences_that_share_a_state(fs, L):
    """One state that several sequences begin with, and one that has none: the sum of their gradients, in their order."""
    import torch
    c = Case(fs, "f32", 4, 2, 1, L, 32, 48, "slow")
    slots = torch.tensor([1, 1, 5, 1], dtype=torch.int32).cuda()
    start = torch.randn((3, 1, 32, 48), generator=torch.Generator().manual_seed(3)).cuda()
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=start, slots=slots)
    got = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=start, slots=slots)
    total = 0
    for b, at in enumerate((1, 1, None, 1)):
        y, _ = c.forward(b, None if at is None else start[at])
        close(Y[b], y, F32)
        want = c.backward(b, None if at is None else start[at])
        for x, w in zip(got[:3], want):
            close(x[b], w, F32)
        if at is not None:
            total = total + want[3]
    close(got[3][1], total, F32)
    assert (got[3][0] == 0).all() and (got[3][2] == 0).all()
    again = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=start, slots=slots)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


def test_gradients_against_differences(fs):
    """Central differences of the forward call in fp32: sum(Y dY) + sum(after dafter) is linear in each input, so that a difference of step 1 is
    exact up to its rounding, 2^-24 of the sum's terms (a few thousand of size 1)."""
    import torch
    c = Case(fs, "f32", 1, 2, 1, 70, 16, 24, "slow")

    def value(Q, K, V, S):
        after = torch.empty_like(S)
        Y = fs.decay_attention(Q, K, V, c.g, c.s, before=S, after=after)
        return (Y.double() * c.dY.double()).sum() + (after.double() * c.dS.double()).sum()

    args = [c.Q, c.K, c.V, c.S0]
    grads = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=c.S0, dafter=c.dS)
    for i, grad in enumerate(grads):
        direction = torch.randn(args[i].shape, generator=torch.Generator().manual_seed(i)).cuda()
        up, down = ([a if j != i else a + sign * direction for j, a in enumerate(args)] for sign in (1.0, -1.0))
        up[i], down[i] = (t if i == 3 else fs._empty(t.shape, t.dtype, t.device).copy_(t) for t in (up[i], down[i]))
        want = (value(*up) - value(*down)) / 2
        size = (grad.double() * direction.double()).norm()
        assert abs(float((grad.double() * direction.double()).sum() - want)) <= 1e-4 * float(size) + 1e-3


# ------------------------------------------------------------------------------------------------ numbers that are not finite
@pytest.mark.parametrize("dtype,d,L", [("bf16", 64, 330), ("bf16", 128, 330), ("f32", 128, 330), ("f32", 32, 1300), ("bf16", 64, 1300)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_numbers_that_are_not_finite_stay_in_their_chunk_and_behind_it(fs, dtype, d, L, bad):
    """Rows of chunks before the one with the number, other heads and sequences: bit for bit as without it; gradients of rows behind its chunk,
    too (they are summed from the last row on)."""
    import torch
    c = Case(fs, dtype, 2, 4, 2, L, d, d, "slow")
    t = [x.clone() for x in (c.Q, c.K, c.V, c.dY)]
    row = 200
    for which in (1, 2, 3):
        with_it = [x.clone() for x in t]
        with_it[which][1, 1, row, 3] = bad                   # a key head, or a query head of the first key head
        states = [torch.empty_like(c.S0) for _ in range(2)]
        Y, Z = (fs.decay_attention(*x[:3], c.g, c.s, before=c.S0, after=S) for x, S in zip((t, with_it), states))
        got, new = (fs.decay_attention_backward(*x, c.g, c.s, before=c.S0) for x in (t, with_it))
        assert torch.equal(Y[0], Z[0]) and torch.equal(states[0][0], states[1][0])
        assert all(torch.equal(x[0], y[0]) for x, y in zip(got, new))
        first = row // 64 * 64
        assert torch.equal(Y[1, :, :first], Z[1, :, :first])
        other = 0 if which < 3 else 1                         # a key head without the number, and its query heads
        q = slice(2 * other, 2 * other + 2)
        assert torch.equal(Y[1, q], Z[1, q]) and torch.equal(states[0][1, other], states[1][1, other])
        assert torch.equal(got[0][1, q], new[0][1, q]) and all(torch.equal(x[1, other], y[1, other]) for x, y in zip(got[1:], new[1:]))
        if which < 3:
            assert not Z[1, 2:, row].isfinite().all() and torch.equal(got[0][1, :, :first], new[0][1, :, :first])
        else:
            # the walk from the last row counts its chunks, and those of its segments, from there
            after = slice(row + 64, L)
            assert all(torch.equal(x[1, :, after], y[1, :, after]) for x, y in zip(got[1:3], new[1:3]))
            assert not new[2][1, 0, :row].isfinite().all()


# ------------------------------------------------------------------------------------------------ strides, streams, graphs, workspaces
def test_strides(fs):
    """Rows of [B, L, heads, d] tensors, one packed tensor of queries, keys and values, outputs in the same layout."""
    import torch
    gen = torch.Generator().manual_seed(4)
    B, L, H, Hk, d = 2, 150, 4, 2, 64
    packed = torch.randn((B, L, H + 2 * Hk, d), generator=gen).bfloat16().cuda()
    Q, K, V = (t.transpose(1, 2) for t in packed.split([H, Hk, Hk], dim=2))
    out = torch.full((B, L, H + 1, d), 5.0, dtype=torch.bfloat16, device="cuda")
    g = decays("slow", Hk).cuda()
    Y = fs.decay_attention(Q, K, V, g, 0.3, out=out[:, :, :H].transpose(1, 2))
    assert torch.equal(Y, fs.decay_attention(Q.contiguous(), K.contiguous(), V.contiguous(), g, 0.3)) and (out[:, :, H] == 5.0).all()
    dY = torch.randn((B, L, H, d), generator=gen).bfloat16().cuda().transpose(1, 2)
    grads = torch.full_like(packed, math.nan)
    got = fs.decay_attention_backward(Q, K, V, dY, g, 0.3, grads=[t.transpose(1, 2) for t in grads.split([H, Hk, Hk], dim=2)])
    want = fs.decay_attention_backward(Q.contiguous(), K.contiguous(), V.contiguous(), dY.contiguous(), g, 0.3)
    assert all(torch.equal(x, y) for x, y in zip(got[:3], want[:3])) and grads.isfinite().all()
    one = K[:, :1, :, :].expand(B, Hk, L, d)              # a broadcast head
    close(fs.decay_attention(Q, one, V, g, 0.3), fs.decay_attention(Q, one.contiguous(), V, g, 0.3).cpu(), 0.0)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 128)])
def test_graphs_streams_and_workspaces(fs, dtype, d):
    """Captured calls replayed on other inputs, with eager work between; two graphs that share a workspace; the ends of a workspace."""
    import torch
    c = Case(fs, dtype, 1, 4, 2, 900, d, d, "slow")
    need = max(fs.lib().favorsharp_decay_attention_workspace_bytes(1, 4, 2, 900, d, d),
               fs.lib().favorsharp_decay_attention_backward_workspace_bytes(1, 4, 2, 900, d, d, 1))
    assert need > 0
    room = torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")
    ws = room[256:256 + need]
    Q, K, V, dY, S0 = (t.clone() for t in (c.Q, c.K, c.V, c.dY, c.S0))
    slots = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = {}

    def forward_call():
        after = torch.empty_like(S0)
        return fs.decay_attention(Q, K, V, c.g, c.s, before=S0, after=after, workspace=ws), after

    def backward_call():
        return fs.decay_attention_backward(Q, K, V, dY, c.g, c.s, before=S0, slots=slots, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        forward_call(), backward_call()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for name, call in (("y", forward_call), ("g", backward_call)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out[name] = call()
        graphs.append(graph)
    for i in range(4):
        gen = torch.Generator().manual_seed(50 + i)
        for t in (Q, K, V, dY, S0):
            t.copy_(torch.randn(t.shape, generator=gen).to(t.dtype))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = [t.clone() for t in forward_call() + tuple(backward_call())]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out["y"] + tuple(out["g"]), want))
    assert (room[:256] == 77).all() and (room[256 + need:] == 77).all()
    with pytest.raises(fs.FavorSharpError, match="status 4"):
        fs.decay_attention_backward(Q, K, V, dY, c.g, c.s, before=S0, slots=slots, workspace=ws[:need - 256])


def test_what_lies_around_the_results(fs):
    """Rows of other tensors beside the results, states beside the pool's: as they were."""
    import torch
    c = Case(fs, "bf16", 2, 2, 2, 67, 24, 40, "slow")
    out = torch.full((2, 4, 70, 48), 9.0, dtype=torch.bfloat16, device="cuda")
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, out=out[:, 1:3, 1:68, :40])
    kept = out.clone()
    kept[:, 1:3, 1:68, :40] = 9.0
    assert (kept == 9.0).all()
    for b in range(2):
        close(Y[b], c.forward(b)[0], BF16)


# ------------------------------------------------------------------------------------------------ heads that share states, in place
@pytest.mark.parametrize("dtype,B,H,Hk,L,d,dv", [("bf16", 60, 24, 8, 1, 64, 64), ("bf16", 60, 24, 8, 64, 64, 64), ("f32", 45, 12, 4, 64, 128, 128), ("bf16", 63, 32, 8, 200, 64, 40),
                                                 ("bf16", 16, 64, 8, 190, 128, 128), ("f32", 60, 64, 8, 33, 24, 33)])
def test_in_place_is_as_into_another_pool(fs, dtype, B, H, Hk, L, d, dv):
    """More workgroups than the chip holds, whose heads read the states that the call goes on from: bit for bit what a call into another pool
    gives, with a padded batch, a sequence without a slot and one that has another's."""
    import torch
    c = Case(fs, dtype, B, H, Hk, L, d, dv, "slow", [L if b % 3 else 1 + b * L // (2 * B) for b in range(B)])
    slots = torch.randperm(B + 2, generator=torch.Generator().manual_seed(B)).to(torch.int32)[:B]
    slots[3], slots[5] = -1, slots[2]
    slots = slots.cuda()
    start = torch.randn((B + 2, Hk, d, dv), generator=torch.Generator().manual_seed(L)).cuda()
    other, counts = start.clone(), torch.zeros(2, dtype=torch.int32, device="cuda")
    want = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=start, after=other, lengths=c.lengths, slots=slots, left_out=counts[:1])
    room = fs.lib().favorsharp_decay_attention_workspace_bytes(B, H, Hk, L, d, dv)
    ws = torch.full((room + 256,), 77, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        pool = start.clone()
        got = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=pool, after=pool, lengths=c.lengths, slots=slots, left_out=counts[1:], workspace=ws[:room])
        assert torch.equal(got, want) and torch.equal(pool, other)
    assert counts.tolist() == [2, 6] and (ws[room:] == 77).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 96)])
def test_shared_heads_in_place(fs, dtype, d):
    """Sequences of 1 to 190 rows, eight query heads to a key head: every head and state against the recurrence, eager and replayed."""
    import torch
    B, H, Hk, L = 16, 32, 4, 190
    c = Case(fs, dtype, B, H, Hk, L, d, d, "slow", [1 + (b * 63) % L for b in range(B)])
    pool = c.S0.clone()
    call = lambda: fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=pool, after=pool, lengths=c.lengths)      # noqa: E731
    Y = call()
    for b in range(B):
        y, S = c.forward(b, c.S0[b])
        close(Y[b], y, tolerance(dtype))
        close(pool[b], S, F32)
    end = pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for _ in range(3):
        pool.copy_(c.S0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, Y) and torch.equal(pool, end)
