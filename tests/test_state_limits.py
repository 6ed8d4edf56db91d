"""The largest calls that the header allows, and the next ones: refused before any launch.  No GPU."""
import pytest

from .test_state_abi import A, P, append, features, fs, pool, tensor  # noqa: F401 (fs: a fixture)


@pytest.mark.parametrize("B,L", [(1, 1 << 28), (8, 1 << 25), (9, 1 << 24)])
def test_more_angles_than_a_launch_has_threads(fs, B, L):  # noqa: F811
    rot = fs.FsRotary(A, None, 0, 0, 64, 0, 1.0)
    lib, f, s, t, ds = fs.lib(), features(fs), pool(fs), tensor(fs), pool(fs, shift=None)
    ws = (A, 1 << 60, None)
    assert B * L * 32 > (1 << 32) - 256
    assert append(fs, B=B, L=L, rot=P(rot), nbytes=1 << 60) == 2
    assert lib.favorsharp_state_attention(P(f), P(s), None, P(t), B, 2, L, 64, None, P(rot), P(t), None, *ws) == 2
    assert lib.favorsharp_state_attention_backward(P(f), P(s), None, P(t), P(t), B, 2, L, 64, None, P(rot), P(t), P(ds), *ws) == 2
    assert lib.favorsharp_state_append_backward(P(f), P(s), None, P(ds), P(t), P(t), B, L, 64, None, P(rot), P(t), P(t), *ws) == 2


def test_more_rows_than_a_launch_has_threads(fs):  # noqa: F811
    rot = fs.FsRotary(A, None, 0, 0, 16, 0, 1.0)
    t, u = tensor(fs, d=1024), tensor(fs, d=1024, ptr=2 * A)
    def call(B, L, d):
        return fs.lib().favorsharp_rotary(P(rot), P(t), 1, None, 0, B, L, d, 0, P(u), None, None)
    assert call(1 << 16, (1 << 15) + 1, 16) == 2                # B L beyond 2^31
    assert call(1 << 10, 1 << 16, 1024) == 2                    # 2^26 rows of 127 threads
