"""Linear attention with a decay and rotary positions with several axes: what the entry points refuse before any device work, sizes,
sections.  No GPU."""
import ctypes
import math

import numpy as np
import pytest

from .test_state_abi import A, P, fs, tensor  # noqa: F401 (fs: a fixture)

OK, INVALID, UNSUPPORTED, SMALL = 0, 1, 2, 4


def pool(fs, S=A, slots=4):  # noqa: F811
    return fs.FsDecayState(S, slots)


def forward(fs, Q=None, K=None, V=None, Y=None, B=2, H=4, heads=2, L=8, d=64, dv=64, g=A, scale=1.0, before=None, after=None, slots=None,  # noqa: F811
            lengths=None, left_out=None, ws=A, nbytes=1 << 40):
    Q, K, V, Y = (t or tensor(fs) for t in (Q, K, V, Y))
    return fs.lib().favorsharp_decay_attention(P(Q), P(K), P(V), B, H, heads, L, d, dv, g, scale, before and P(before), after and P(after), slots,
                                               lengths, P(Y), left_out, ws, nbytes, None)


def backward(fs, Q=None, dY=None, dQ=None, L=8, before=None, dafter=None, dbefore=None, exclusive=0, ws=A, nbytes=1 << 40, scale=1.0, B=2, d=64):  # noqa: F811
    Q, dY, dQ, t = Q or tensor(fs), dY or tensor(fs), dQ or tensor(fs), tensor(fs)
    return fs.lib().favorsharp_decay_attention_backward(P(Q), P(t), P(t), P(dY), B, 4, 2, L, d, 64, A, scale, before and P(before), dafter and P(dafter),
                                                        None, None, exclusive, P(dQ), P(t), P(t), dbefore and P(dbefore), ws, nbytes, None)


def step(fs, state=None, Q=None, Y=None, B=2, H=4, heads=2, d=64, dv=64, g=A, scale=1.0):  # noqa: F811
    Q, Y, t = Q or tensor(fs), Y or tensor(fs), tensor(fs)
    return fs.lib().favorsharp_decay_step(P(state or pool(fs)), None, P(Q), P(t), P(t), B, H, heads, d, dv, g, scale, P(Y), None, None)


def test_rows_are_refused(fs):  # noqa: F811
    for bad in (dict(B=0), dict(L=-1), dict(H=3), dict(heads=0), dict(H=0), dict(d=0), dict(dv=0), dict(g=None), dict(g=A + 2), dict(scale=math.inf),
                dict(scale=math.nan), dict(Q=tensor(fs, ptr=None)), dict(K=tensor(fs, ptr=A + 2)), dict(V=tensor(fs, dtype=0)), dict(Y=tensor(fs, stride=60)),
                dict(Q=tensor(fs, dtype=3)), dict(before=pool(fs, S=None)), dict(after=pool(fs, S=A + 4)), dict(before=pool(fs, slots=0)),
                dict(before=pool(fs), after=pool(fs, slots=5)), dict(slots=A + 1), dict(lengths=A + 2), dict(left_out=A + 1), dict(ws=A + 4)):
        assert forward(fs, **bad) == INVALID, bad
    for bad in (dict(d=129), dict(dv=129, V=tensor(fs, 136), Y=tensor(fs, 136)), dict(B=40000), dict(L=1 << 29), dict(before=pool(fs, slots=40000))):
        bad.setdefault("Q", tensor(fs, 136)), bad.setdefault("K", tensor(fs, 136))
        assert forward(fs, **bad) == UNSUPPORTED, bad
    assert forward(fs, L=0) == OK                       # nothing to do
    assert forward(fs, L=100000, ws=None, nbytes=0) == INVALID
    assert forward(fs, L=100000, nbytes=4096) == SMALL


def test_gradients_are_refused(fs):  # noqa: F811
    for bad in (dict(exclusive=2), dict(exclusive=1), dict(dafter=pool(fs)), dict(dY=tensor(fs, dtype=0)), dict(dQ=tensor(fs, ptr=None)), dict(scale=math.nan),
                dict(before=pool(fs), dbefore=pool(fs, slots=3)), dict(dbefore=pool(fs, S=None)), dict(dbefore=pool(fs), ws=None), dict(ws=A + 8)):
        assert backward(fs, **bad) == INVALID, bad
    assert backward(fs, d=129, Q=tensor(fs, 136), dQ=tensor(fs, 136)) == UNSUPPORTED
    assert backward(fs, dbefore=pool(fs), nbytes=64) == SMALL
    assert backward(fs, L=0) == OK


def test_tokens_are_refused(fs):  # noqa: F811
    for bad in (dict(state=pool(fs, S=None)), dict(B=0), dict(H=3), dict(g=None), dict(scale=math.nan), dict(Q=tensor(fs, dtype=0)), dict(Y=tensor(fs, ptr=None))):
        assert step(fs, **bad) == INVALID, bad
    assert step(fs, d=129, Q=tensor(fs, 136)) == UNSUPPORTED
    assert step(fs, B=40000) == UNSUPPORTED
    assert fs.lib().favorsharp_decay_step(None, None, P(tensor(fs)), P(tensor(fs)), P(tensor(fs)), 1, 1, 1, 64, 64, A, 1.0, P(tensor(fs)), None, None) == INVALID


def test_workspaces(fs):  # noqa: F811
    f, b = fs.lib().favorsharp_decay_attention_workspace_bytes, fs.lib().favorsharp_decay_attention_backward_workspace_bytes
    assert f(4096, 8, 8, 1024, 64, 64) == 0 and f(1, 8, 8, 64, 64, 64) == 0          # one segment
    assert f(1, 8, 8, 16384, 64, 64) >= 2 * 8 * 64 * 64 * 4
    assert f(1, 8, 3, 16384, 64, 64) == f(1, 8, 8, 16384, 129, 64) == f(70000, 1, 1, 16, 64, 64) == 0
    assert b(4096, 8, 8, 128, 64, 64, 0) == 0 and b(4096, 8, 8, 128, 64, 64, 1) >= 4096 * 8 * 64 * 64 * 4
    assert b(1, 8, 8, 16384, 64, 64, 0) >= 2 * 2 * 8 * 64 * 64 * 4
    assert b(1, 8, 3, 16384, 64, 64, 1) == 0


def test_rotary_axes_refuses(fs):  # noqa: F811
    t, u = tensor(fs), tensor(fs, ptr=2 * A)

    def call(freqs=A, axis_of=A, positions=A, sa=8, sb=8, sl=1, axes=3, rot=64, interleaved=0, amplitude=1.0, d=64, X=t, Y=u, L=4, none=False):
        r = fs.FsRotaryAxes(freqs, axis_of, positions, sa, sb, sl, axes, rot, interleaved, amplitude)
        return fs.lib().favorsharp_rotary_axes(None if none else P(r), P(X), 2, None, 0, 1, L, d, 0, P(Y), None, None)

    for bad in (dict(freqs=None), dict(axis_of=None), dict(positions=None), dict(axis_of=A + 2), dict(positions=A + 1), dict(sa=-1), dict(sb=-1), dict(sl=-1),
                dict(axes=0), dict(axes=9), dict(rot=63), dict(rot=0), dict(rot=66), dict(interleaved=2), dict(amplitude=math.inf), dict(none=True),
                dict(L=-1), dict(Y=tensor(fs, stride=128))):
        assert call(**bad) == INVALID, bad
    assert call(L=0) == OK
    assert call(d=1032, X=tensor(fs, 1032), Y=tensor(fs, 1032, ptr=2 * A)) == UNSUPPORTED


def test_sections(fs):  # noqa: F811
    f, a = fs.rotary_sections([4, 2, 2], device="cpu")
    assert a.tolist() == [0, 0, 0, 0, 1, 1, 2, 2]
    np.testing.assert_allclose(f.numpy(), [1e4 ** -(i / n) for n in (4, 2, 2) for i in range(n)], rtol=1e-14)
    f, a = fs.rotary_sections([4, 1, 3], base=100.0, order="cyclic", whole=True, device="cpu")
    assert a.tolist() == [0, 1, 2, 0, 2, 0, 2, 0]
    np.testing.assert_allclose(f.numpy(), [100.0 ** -(i / 8) for i in range(8)], rtol=1e-14)
    f, a = fs.rotary_sections([2, 0, 1], order="cyclic", device="cpu")
    assert a.tolist() == [0, 2, 0] and f.tolist() == [1.0, 1.0, 0.01]
    np.testing.assert_allclose(fs.rotary_sections([16], device="cpu")[0], fs.rotary_frequencies(32, device="cpu"), rtol=1e-14)      # one axis
    for bad in (dict(pairs=[]), dict(pairs=[0, 0]), dict(pairs=[-1, 2]), dict(pairs=[500, 13]), dict(pairs=[1] * 9), dict(pairs=[4], base=1.0)):
        with pytest.raises(fs.FavorSharpError):
            fs.rotary_sections(device="cpu", **bad)
    with pytest.raises(KeyError):
        fs.rotary_sections([4], order="other", device="cpu")


def test_positions_with_several_axes_are_for_rotary_alone(fs):  # noqa: F811
    import torch
    with pytest.raises(TypeError, match="rotary"):
        fs._rotary_desc(fs.RotaryAxes(torch.ones(4, dtype=torch.float64), torch.zeros(4, dtype=torch.int32), torch.zeros(2, 8, dtype=torch.int32)), 1, 8)


def test_tensors_of_the_host_are_refused(fs):  # noqa: F811
    import torch
    t, g = torch.zeros(1, 2, 4, 8), torch.zeros(2)
    with pytest.raises(ValueError, match="device"):
        fs.decay_attention(t, t, t, g)
    with pytest.raises(ValueError, match="shape"):
        fs.decay_attention(t, t[:, :, :3], t, g)
    with pytest.raises(ValueError, match="shape"):
        fs.decay_step(torch.zeros(1, 2, 8, 8), t, t, t, g)
    with pytest.raises(ValueError, match="slots"):
        fs.decay_step(torch.zeros(1, 2, 8, 8), *[torch.zeros(2, 2, 1, 8)] * 3, g)
    with pytest.raises(ValueError, match="float32"):
        fs.decay_attention(t, t, t, g, before=torch.zeros(1, 2, 8, 8).half())
    with pytest.raises(ValueError, match="shape"):
        fs.decay_attention(t, t, t, torch.zeros(3))
    with pytest.raises(ValueError, match="shape"):
        fs.decay_attention(t, t, t, g, before=torch.zeros(3, 2, 8, 8), after=torch.zeros(2, 2, 8, 8))
    with pytest.raises(ValueError, match="shape"):
        fs.decay_attention_backward(t, t, t, t[..., :4], g)


@pytest.mark.parametrize("B,H,heads,L,d,dv", [(60, 24, 8, 64, 64, 64), (60, 24, 8, 1, 64, 64), (45, 12, 4, 64, 128, 128), (16, 64, 8, 190, 128, 128), (1, 2, 1, 1, 8, 8),
                                              (63, 16, 8, 448, 64, 64), (3, 4, 2, 0, 64, 40)])
def test_shared_heads_in_place_keep_their_states_apart(fs, B, H, heads, L, d, dv):  # noqa: F811
    """One segment, query heads in workgroups of their own: none of them may write the pool that the others read, so the states after an
    in-place call need a workspace."""
    need = fs.lib().favorsharp_decay_attention_workspace_bytes(B, H, heads, L, d, dv)
    assert need >= B * heads * d * dv * 4
    t = tensor(fs, 128)
    for nbytes, ws, want in ((0, None, INVALID), (need - 1, A, SMALL)):
        assert forward(fs, t, t, t, t, B, H, heads, L, d, dv, before=pool(fs, slots=B), after=pool(fs, slots=B), ws=ws, nbytes=nbytes) == want
    assert fs.lib().favorsharp_decay_attention_workspace_bytes(B, heads, heads, min(L, 64), d, dv) == 0       # heads of their own
