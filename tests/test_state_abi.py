"""Entry points on kept states and rotary positions: what they refuse before any device work, sizes, frequencies.  No GPU."""
import ctypes
import math

import numpy as np
import pytest


@pytest.fixture(scope="module")
def fs():
    import os
    from paper_2302_00787_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2302_00787_amd import build
        build.build(verbose=False)
    binding.lib()
    return binding


P = ctypes.byref
A = 1 << 20        # an address that is aligned and never read here


def features(fs, heads=2, d=64, M=256, sets=2, dense=0, nbytes=1 << 30, ptr=A):
    return fs.FsFeatures(ptr, nbytes, heads, d, M, sets, dense, 0.35)


def tensor(fs, d=64, ptr=A, dtype=1, stride=None):
    return fs.FsTensor(ptr, dtype, 1024, 512, stride or d)


def pool(fs, T=A, z=A, shift=A, slots=4):
    return fs.FsState(T, z, shift, slots)


def append(fs, f=None, s=None, K=None, V=None, B=2, L=8, dv=64, rot=None, fresh=0, ws=A, nbytes=1 << 30):
    f, s, K, V = f or features(fs), s or pool(fs), K or tensor(fs), V or tensor(fs)
    return fs.lib().favorsharp_state_append(P(f), P(s), None, P(K), P(V), B, L, dv, None, rot, fresh, None, ws, nbytes, None)


def test_append_refuses(fs):
    assert append(fs, f=features(fs, ptr=None)) == 1
    assert append(fs, f=features(fs, sets=3)) == 1
    assert append(fs, f=features(fs, dense=2)) == 1
    assert append(fs, f=features(fs, d=129)) == 2
    assert append(fs, f=features(fs, M=2049)) == 2
    assert append(fs, f=features(fs, nbytes=1024)) == 4
    assert append(fs, s=pool(fs, T=None)) == 1
    assert append(fs, s=pool(fs, T=A + 4)) == 1
    assert append(fs, s=pool(fs, shift=None)) == 1
    assert append(fs, s=pool(fs, slots=0)) == 1
    assert append(fs, s=pool(fs, slots=40000)) == 2
    assert append(fs, B=0) == 1
    assert append(fs, L=-1) == 1
    assert append(fs, dv=129, V=tensor(fs, 136)) == 2
    assert append(fs, B=40000) == 2
    assert append(fs, K=tensor(fs, ptr=None)) == 1
    assert append(fs, K=tensor(fs, ptr=A + 2)) == 1
    assert append(fs, K=tensor(fs, stride=60)) == 1
    assert append(fs, V=tensor(fs, dtype=0)) == 1
    assert append(fs, K=tensor(fs, dtype=7)) == 1
    assert append(fs, fresh=2) == 1
    assert append(fs, ws=None) == 1
    assert append(fs, ws=A + 4) == 1
    assert append(fs, nbytes=1024) == 4
    for rot in (fs.FsRotary(None, None, 0, 0, 64, 0, 1.0), fs.FsRotary(A, None, 0, 0, 63, 0, 1.0), fs.FsRotary(A, None, 0, 0, 66, 0, 1.0),
                fs.FsRotary(A, None, 0, 0, 0, 0, 1.0), fs.FsRotary(A, None, -1, 0, 64, 0, 1.0), fs.FsRotary(A, None, 0, 0, 64, 2, 1.0),
                fs.FsRotary(A, None, 0, 0, 64, 0, math.inf), fs.FsRotary(A, A + 1, 0, 0, 64, 0, 1.0)):
        assert append(fs, rot=P(rot)) == 1


def test_the_other_entry_points_refuse(fs):
    L = fs.lib()
    f, s, t, ds = features(fs), pool(fs), tensor(fs), pool(fs, shift=None)
    ws = (A, 1 << 30, None)
    # query heads that are no multiple of the key heads; a pool of gradients with other slots; null tensors
    assert L.favorsharp_state_attention(P(f), P(s), None, P(t), 2, 3, 8, 64, None, None, P(t), None, *ws) == 1
    assert L.favorsharp_state_attention(P(f), P(s), None, None, 2, 4, 8, 64, None, None, P(t), None, *ws) == 1
    rot = fs.FsRotary(A, None, 0, 0, 64, 0, 1.0)
    assert L.favorsharp_state_attention(P(f), P(s), None, P(t), 2, 4, 8, 64, None, P(rot), P(t), None, A, 0, None) == 4
    assert L.favorsharp_state_attention(P(f), P(s), None, P(t), 2, 4, 8, 64, None, P(rot), P(t), None, None, 1 << 20, None) == 1
    assert L.favorsharp_state_attention(P(f), P(s), None, P(t), 2, 4, 8, 64, None, None, None, None, *ws) == 1
    assert L.favorsharp_state_step(P(f), P(s), None, P(t), P(t), P(t), 2, 3, 64, None, P(t), None, *ws) == 1
    assert L.favorsharp_state_step(P(f), P(s), None, P(t), P(tensor(fs, dtype=0)), P(t), 2, 4, 64, None, P(t), None, *ws) == 1
    assert L.favorsharp_state_step(P(f), P(s), None, P(t), P(t), P(t), 128, 4, 64, None, P(t), None, A, 512, None) == 4
    assert L.favorsharp_state_step(P(f), P(s), None, P(t), P(t), P(t), 128, 4, 64, None, P(t), None, None, 1 << 30, None) == 1
    assert L.favorsharp_state_attention_backward(P(f), P(s), None, P(t), P(t), 2, 4, 8, 64, None, None, P(t), P(pool(fs, slots=5)), *ws) == 1
    assert L.favorsharp_state_attention_backward(P(f), P(s), None, P(t), P(t), 2, 4, 8, 64, None, None, None, P(ds), *ws) == 1
    assert L.favorsharp_state_attention_backward(P(f), P(s), None, P(t), P(t), 2, 4, 8, 64, None, None, P(t), P(ds), A, 1000, None) == 4
    assert L.favorsharp_state_append_backward(P(f), P(s), None, P(pool(fs, z=None)), P(t), P(t), 2, 8, 64, None, None, P(t), P(t), *ws) == 1
    assert L.favorsharp_state_append_backward(P(f), P(s), None, P(ds), P(t), P(t), 2, 8, 64, None, None, P(t), None, *ws) == 1
    rot = fs.FsRotary(A, None, 0, 0, 64, 0, 1.0)
    assert L.favorsharp_state_append_backward(P(f), P(s), None, P(ds), P(t), P(t), 2, 8, 64, None, P(rot), P(t), P(t), A, 8, None) == 4
    # more rows of a state than are counted in 32 bits
    assert L.favorsharp_state_attention(P(f), P(s), None, P(t), 1, 8, 1 << 28, 64, None, None, P(t), None, *ws) == 2
    # nothing to do
    assert L.favorsharp_state_attention(P(f), P(s), None, P(t), 2, 4, 0, 64, None, None, P(t), None, *ws) == 0
    assert L.favorsharp_state_prepare(None, 1, A, 1, 1, 64, 256, 1.0, P(features(fs)), None) == 1
    assert L.favorsharp_state_prepare(A, 3, A, 1, 2, 64, 256, 1.0, P(features(fs)), None) == 1
    assert L.favorsharp_state_prepare(A, 1, A, 1, 2, 129, 256, 1.0, P(features(fs)), None) == 2
    assert L.favorsharp_state_prepare(A, 1, A, 1, 2, 64, 256, 1.0, P(features(fs, nbytes=1024)), None) == 4


def test_rotary_refuses(fs):
    L = fs.lib()
    r, t, u = fs.FsRotary(A, None, 0, 0, 64, 0, 1.0), tensor(fs), tensor(fs, ptr=2 * A)
    def call(r=r, X=t, H=2, X2=None, H2=0, B=1, n=4, d=64, back=0, Y=u, Y2=None):
        return L.favorsharp_rotary(None if r is None else P(r), P(X) if X else None, H, P(X2) if X2 else None, H2, B, n, d, back,
                                   P(Y) if Y else None, P(Y2) if Y2 else None, None)
    assert call(r=None) == call(X=None) == call(Y=None) == call(back=2) == call(H=0) == call(B=0) == call(n=-1) == 1
    assert call(d=62) == 1                                  # rot_dim > d
    assert call(X2=u, H2=1) == 1                            # no second output
    assert call(Y=tensor(fs, stride=128)) == 1              # in place on other strides
    assert call(Y=tensor(fs, dtype=0)) == 1
    assert call(n=0) == 0
    assert call(d=1032, X=tensor(fs, 1032), Y=tensor(fs, 1032, ptr=2 * A)) == 2


def test_workspace_sizes(fs):
    L = fs.lib()
    f = features(fs)
    state = 256 * 65 * 4
    n = L.favorsharp_state_append_workspace_bytes(P(f), 4, 4096, 64, 0)
    assert n >= 4 * 2 * state
    assert L.favorsharp_state_append_workspace_bytes(P(f), 4, 4096, 64, 64) >= n + 4 * 4096 * 32 * 8        # the angles
    assert L.favorsharp_state_append_workspace_bytes(P(features(fs, dense=1)), 4, 4096, 64, 0) >= n + 8 * 4096 * 4
    assert L.favorsharp_state_attention_workspace_bytes(P(f), 4, 4, 4096, 64, 0) == 0             # nothing is kept between launches
    assert L.favorsharp_state_attention_workspace_bytes(P(f), 4, 4, 4096, 64, 64) >= 4 * 4096 * 32 * 8
    assert L.favorsharp_state_attention_backward_workspace_bytes(P(f), 4, 4, 4096, 64, 0) >= 16 * 4096 * 8 + 8 * state
    assert L.favorsharp_state_append_backward_workspace_bytes(P(f), 4, 4096, 64, 0) == 0
    assert L.favorsharp_state_append_backward_workspace_bytes(P(f), 4, 4096, 64, 64) >= 4 * 4096 * 32 * 8
    assert L.favorsharp_state_append_workspace_bytes(None, 4, 4096, 64, 0) == 0
    assert L.favorsharp_state_append_workspace_bytes(P(f), 4, 4096, 129, 0) == 0
    assert L.favorsharp_state_attention_workspace_bytes(P(f), 4, 3, 4096, 64, 0) == 0
    assert L.favorsharp_state_step_workspace_bytes(P(f), 4, 2) == 0                                # one launch
    assert L.favorsharp_state_step_workspace_bytes(P(f), 256, 4) >= 256 * (4 + 2 + 2) * 256 * 4
    assert L.favorsharp_state_features_bytes(2, 64, 256, 1, 2) > 2 * 2 * 256 * 64 * (4 + 6)
    assert L.favorsharp_state_features_bytes(2, 64, 256, 3, 2) == L.favorsharp_state_features_bytes(2, 64, 4000, 1, 1) == 0


def test_rotary_frequencies(fs):
    n, base = 64, 10000.0
    i = np.arange(n // 2)
    plain = base ** (-2.0 * i / n)
    f = lambda **k: fs.rotary_frequencies(n, device="cpu", **k).numpy()
    np.testing.assert_allclose(f(), plain, rtol=1e-14)
    np.testing.assert_allclose(f(scaling="linear", factor=4.0), plain / 4, rtol=1e-14)
    b = f(scaling="base", factor=4.0)
    assert b[0] == 1.0 and abs(b[-1] * 4 / plain[-1] - 1) < 1e-12
    c = f(scaling="blend", factor=4.0, original_length=4096)
    turns = 4096 * plain / (2 * math.pi)
    np.testing.assert_allclose(c[turns >= 32], plain[turns >= 32], rtol=1e-14)
    np.testing.assert_allclose(c[turns <= 1], plain[turns <= 1] / 4, rtol=1e-14)
    assert ((c <= plain * (1 + 1e-14)) & (c >= plain / 4 * (1 - 1e-14))).all() and (np.diff(c) < 0).all()
    assert fs.rotary_frequencies(2, scaling="base", factor=2.0, device="cpu").tolist() == [1.0]
    for bad in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=64, base=1.0), dict(rot_dim=64, base=math.nan), dict(rot_dim=64, scaling="linear", factor=0.0),
                dict(rot_dim=64, scaling="linear", factor=math.inf), dict(rot_dim=64, scaling="blend", factor=2.0, original_length=0),
                dict(rot_dim=64, scaling="blend", factor=2.0, original_length=8, low_turns=4.0, high_turns=4.0)):
        with pytest.raises(fs.FavorSharpError):
            fs.rotary_frequencies(device="cpu", **bad)
