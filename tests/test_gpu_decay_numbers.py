"""Linear attention with a decay for each head: numbers besides the everyday ones.

States that are far larger than what is read of them: S = `MEAN` + ordinary numbers, and rows whose pairs of numbers cancel, (x, -x), so that the mean
leaves nothing and the terms of a sum are far larger than the sum.  Sums and products are fp32's.  A state that a second chunk reads was decayed
once and added to by six products (a chunk's 64 rows in two steps, three pieces each), a read adds at most twelve (128 numbers in four steps, three
pieces each): 19 roundings of at most 2^-24 of the terms' size, each in its own direction, 4.4 of them together: twice that, 2^-21 of the root
of the terms' sum of squares (`parts`), is the bar.  Two bf16 pieces of a state would be off by up to 2^-18 of it.  A result rounded to bf16
is off by up to half a step, 2^-8 of the power of two below it, and so by 2^-8 / sqrt(3) of the norm.
"""
import math

import pytest

from .test_gpu_decay import F32, Case, close, fs  # noqa: F401 (fs: a fixture)

pytestmark = pytest.mark.gpu

ROUNDED = 2.0 ** -8 / math.sqrt(3.0)
MEAN = 22962.0               # (22912 has eight bits, and the 50 that it leaves are far larger than the ordinary numbers, too)


@pytest.mark.parametrize("B,H,Hk,L,d,dv", [(1, 2, 2, 100, 64, 64), (2, 4, 2, 100, 128, 128), (1, 2, 1, 100, 32, 32), (1, 2, 2, 100, 128, 64), (1, 4, 2, 90, 64, 128),
                                           (1, 2, 2, 70, 24, 40), (1, 4, 1, 70, 66, 34), (64, 8, 8, 100, 64, 64), (130, 8, 4, 80, 64, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_states_far_larger_than_what_is_read_of_them(fs, dtype, B, H, Hk, L, d, dv):  # noqa: F811
    import torch
    c = Case(fs, dtype, B, H, Hk, L, d, dv, "slow")
    for t in (c.Q, c.K, c.V, c.dY):
        t[..., 1::2] = -t[..., 0::2]
    c.S0 += MEAN
    c.dS += MEAN
    after = torch.empty_like(c.S0)
    Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=c.S0, after=after, out_dtype=torch.bfloat16)
    got = (Y,) + fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=c.S0, dafter=c.dS, grad_dtype=torch.bfloat16)
    i = torch.arange(L, dtype=torch.float64)
    before = torch.exp(c.g.double().cpu()[:, None] * (i + 1))[..., None]               # what is left of the states at each row
    behind = torch.exp(c.g.double().cpu()[:, None] * (L - 1 - i))[..., None]
    for b in (range(B) if B < 9 else (0, B // 2, B - 1)):
        y, S = c.forward(b, c.S0[b])
        want = (y,) + c.backward(b, c.S0[b], c.dS[b])
        close(after[b], S, F32)
        close(got[4][b], want[4], F32)
        q, k, v, dy, _, _ = c.host(b)
        far = before.repeat_interleave(H // Hk, 0)
        parts = [x.norm() * MEAN * math.sqrt(n) for x, n in ((c.s * far * q, dv), (c.s * far * dy, d), (behind * v, d), (behind * k, dv))]
        for name, x, w, part in zip(("Y", "dQ", "dK", "dV"), got, want, parts):
            off, norm = float((x[b].double().cpu() - w).norm()), float(w.norm())
            assert off <= ROUNDED * norm + 2.0 ** -21 * float(part), (name, b, off / norm, float(part) / norm)


@pytest.mark.parametrize("B,H,Hk,L,d,dv", [(1, 2, 2, 300, 64, 64), (2, 4, 2, 130, 128, 128), (1, 2, 1, 900, 64, 96), (1, 4, 1, 1000, 32, 32), (2, 2, 2, 70, 24, 40),
                                           (1, 2, 2, 66, 33, 65), (3, 2, 2, 1500, 128, 64), (64, 8, 8, 200, 64, 64), (1, 4, 2, 1000, 96, 96)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("states", [False, True])
def test_results_differ_by_their_rounding_alone(fs, dtype, B, H, Hk, L, d, dv, states):  # noqa: F811
    """In bf16: those in fp32, rounded."""
    import torch
    c = Case(fs, dtype, B, H, Hk, L, d, dv, "slow", [L - b % 7 for b in range(B)])
    before = c.S0 if states else None
    after = [torch.empty_like(c.S0) if states else None for _ in range(2)]
    both = []
    for dt, S in zip((torch.bfloat16, torch.float32), after):
        Y = fs.decay_attention(c.Q, c.K, c.V, c.g, c.s, before=before, after=S, lengths=c.lengths, out_dtype=dt)
        grads = fs.decay_attention_backward(c.Q, c.K, c.V, c.dY, c.g, c.s, before=before, lengths=c.lengths, grad_dtype=dt)
        both.append((Y, *grads))
    for name, x, y in zip(("Y", "dQ", "dK", "dV"), *both):
        assert x.dtype == torch.bfloat16 and torch.equal(x, y.bfloat16()), name
    if states:
        assert torch.equal(*after) and torch.equal(both[0][4], both[1][4])
