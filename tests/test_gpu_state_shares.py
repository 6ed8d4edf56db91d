"""States of batches that the workgroups share: ragged lengths, sequences without a state, more sequences than a wave counts, more rows than
a grid dimension, and calls that share a workspace.  Against the formulas in 64 bits of test_gpu_state, with its tolerances.
"""
import math

import pytest

from .test_gpu_state import F32, GRAD, Oracle, check, empty_rows, make_rot, make_theta, rows, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fs():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2302_00787_amd import binding
    binding.lib()
    return binding


def oracle(theta, omega, s, heads):
    """Its constants on the GPU."""
    o = Oracle(theta, omega, s, heads)
    for name in ("W1", "W2", "bias", "C2"):
        setattr(o, name, getattr(o, name).cuda())
    return o


def parts_of(o, state, h, dy):
    """For `check` of dq (GRAD, ten times): 2e-5 of what its two parts can be."""
    mean = float((state[0].norm(dim=1) / state[1].clamp_min(1e-300)).max())
    return 1.1 / 50 * dy.norm(dim=1, keepdim=True) * mean * float(o.s * o.W1[h].norm(dim=-1).max())


CASES = [  # d, dv, M, B, heads, group, L, dtype, family, rotation
    # rows in pieces of 256 or more, images in LDS
    (64, 64, 96, 66, 3, 1, 140, "bf16", "iso", None),
    (64, 64, 64, 66, 3, 1, 140, "bf16", "dense", ("half", 1.0)),
    (64, 64, 40, 50, 4, 2, 75, "f32", "dense", ("half", 1.0)),
    (64, 40, 33, 66, 3, 2, 70, "bf16", "iso", ("interleaved", 0.5)),
    (32, 32, 70, 66, 3, 1, 140, "bf16", "dense", None),
    (32, 32, 64, 66, 3, 1, 129, "f32", "iso", ("half", 1.0)),
    (20, 32, 31, 66, 3, 1, 40, "f32", "dense", ("half", 0.3)),
    (128, 128, 64, 66, 3, 1, 70, "bf16", "iso", None),
    (128, 128, 96, 50, 4, 1, 70, "f32", "dense", ("half", 1.0)),
    (96, 128, 50, 66, 3, 1, 40, "bf16", "dense", ("half", 0.5)),
    # few rows; chunks of a padded batch over the workgroups
    (64, 64, 256, 9, 2, 1, 700, "bf16", "iso", ("half", 1.0)),
    (64, 64, 100, 5, 1, 3, 500, "f32", "iso", None),
    (128, 128, 200, 4, 2, 2, 260, "f32", "dense", ("half", 1.0)),
    (128, 100, 520, 3, 1, 2, 300, "bf16", "dense", ("interleaved", 1.0)),
    (24, 16, 600, 6, 8, 1, 333, "bf16", "iso", ("half", 0.5)),
    (64, 64, 64, 6, 2, 1, 300, "bf16", "iso", ("half", 0.5)),
    (32, 32, 512, 5, 3, 1, 77, "f32", "dense", ("half", 0.25)),
    (128, 128, 64, 4, 1, 2, 200, "bf16", "dense", ("half", 0.75)),
    # a workgroup a state
    (32, 32, 40, 300, 1, 1, 200, "bf16", "iso", None),
    (16, 24, 32, 270, 2, 2, 90, "f32", "dense", None),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:9]))
def test_shared_out(fs, case):
    import torch
    d, dv, M, B, heads, G, L, dtype, family, kind = case
    gen = torch.Generator().manual_seed(d + M + B)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    s, H = d ** -0.25, heads * G
    theta, omega = make_theta(gen, family, heads, d), torch.randn((heads, M, d), generator=gen)
    o, f = oracle(theta, omega, s, heads), fs.state_prepare(theta.cuda(), omega.cuda(), s)
    special = torch.tensor([L, 0, 33, 1, 31, 32])[:B // 2]
    n = torch.randint(0, L + 1, (B,), generator=gen)
    n[:len(special)] = special
    n = n[torch.randperm(B, generator=gen)]
    slots = torch.randperm(B + 2, generator=gen)[:B].to(torch.int32)
    if B > 3:
        slots[1], slots[2], slots[3] = -1, B + 2, slots[0]          # none, out of the pool, an earlier one's
    lengths, where = n.to(torch.int32).cuda(), slots.cuda()
    taken = set()
    owner = [i if 0 <= int(x) < B + 2 and not (int(x) in taken or taken.add(int(x))) else -1 for i, x in enumerate(slots)]
    K, V, Q, dY = (rows(gen, dt, B, h, L, c) for h, c in ((heads, d), (heads, dv), (H, d), (H, dv)))
    rot = make_rot(fs, kind, d, B, L, gen)
    k64, q64 = turned(K.double().cpu(), rot).cuda(), turned(Q.double().cpu(), rot).cuda()
    v64, dy64 = V.double(), dY.double()
    for b in range(B):                                              # what is behind a length does not matter
        for t in (K, V, Q, dY):
            t[b, :, int(n[b]):] = float("nan")
    half = L // 2
    state = fs.state_new(B + 2, heads, M, dv)
    left = torch.zeros(1, dtype=torch.int32, device="cuda")
    first = lengths.clamp(max=half)
    rot_a = None if rot is None else rot._replace(positions=rot.positions[:, :half].contiguous())
    rot_b = None if rot is None else rot._replace(positions=rot.positions[:, half:].contiguous())
    fs.state_append(f, state, K[:, :, :half], V[:, :, :half], lengths=first, slots=where, rotary=rot_a, left_out=left)
    fs.state_append(f, state, K[:, :, half:], V[:, :, half:], lengths=lengths - first, slots=where, rotary=rot_b, left_out=left)
    assert int(left) == 2 * sum(i < 0 for i in owner)
    Y = fs.state_attention(f, state, Q, lengths=lengths, slots=where, rotary=rot, out=empty_rows(dt, B, H, L, dv))
    dQ, ds = fs.state_attention_backward(f, state, Q, dY, lengths=lengths, slots=where, rotary=rot)
    gT, gz = (torch.randn(t.shape, generator=gen).cuda() for t in (state.T, state.z))
    dK, dV = fs.state_append_backward(f, state, fs.State(gT, gz, None), K, V, lengths=lengths, slots=where, rotary=rot)
    Yw, dQw = torch.zeros(Y.shape, dtype=torch.float64, device="cuda"), torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    dKw, dVw = torch.zeros(K.shape, dtype=torch.float64, device="cuda"), torch.zeros(V.shape, dtype=torch.float64, device="cuda")
    Tw, zw = torch.zeros(state.T.shape, dtype=torch.float64, device="cuda"), torch.zeros(state.z.shape, dtype=torch.float64, device="cuda")
    dTw, dzw, size = torch.zeros_like(Tw), torch.zeros_like(zw), torch.zeros_like(dQw[..., :1])
    new = (torch.zeros((M, dv), dtype=torch.float64, device="cuda"), torch.zeros(M, dtype=torch.float64, device="cuda"),
           torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
    at = {int(x): i for i, x in enumerate(slots) if owner[i] >= 0}
    readers = {x: [i for i in range(B) if int(slots[i]) == x] for x in at}
    for slot, b in at.items():
        m = int(n[b])
        for h in range(heads):
            st = o.append(new, b, h, k64[b, h, :m], v64[b, h, :m])
            if m:
                assert abs(float(state.shift[slot, h]) - float(st[2])) <= 2e-5
                # (the shift is a largest exponent as the kernel has it: gradients are those of the states with it)
                scale = torch.exp2(st[2] - state.shift[slot, h].double())
                st = (st[0] * scale, st[1] * scale, state.shift[slot, h].double())
            Tw[slot, h], zw[slot, h] = st[0], st[1]
            for i in readers[slot]:                                 # a sequence reads its slot, also if another one wrote it
                r = int(n[i])
                for g in range(G if r else 0):
                    Yw[i, h * G + g, :r] = o.read(st, h, q64[i, h * G + g, :r])
                    dq, dT, dz = o.read_backward(st, h, q64[i, h * G + g, :r], dy64[i, h * G + g, :r])
                    dQw[i, h * G + g, :r] = dq
                    dTw[slot, h] += dT
                    dzw[slot, h] += dz
                    size[i, h * G + g, :r] = parts_of(o, st, h, dy64[i, h * G + g, :r])
    for slot, b in at.items():
        m = int(n[b])
        for h in range(heads if m else 0):
            dKw[b, h, :m], dVw[b, h, :m] = o.append_backward(state.shift[slot, h].double(), h, k64[b, h, :m], v64[b, h, :m], gT[slot, h].double(),
                                                             gz[slot, h].double())
    if rot is not None:
        dQw, dKw = turned(dQw.cpu(), rot, transposed=True).cuda(), turned(dKw.cpu(), rot, transposed=True).cuda()
    check(state.T.flatten(1), Tw.flatten(1).cpu(), F32, "T")
    check(state.z.flatten(1), zw.flatten(1).cpu(), F32, "z")
    check(Y, Yw.cpu(), F32, "Y")
    check(ds.T.reshape(1, -1), dTw.reshape(1, -1).cpu(), F32, "dT")
    check(ds.z.reshape(1, -1), dzw.reshape(1, -1).cpu(), GRAD, "dz")
    check(dQ, dQw.cpu(), GRAD, "dQ", size.cpu())
    check(dK, dKw.cpu(), GRAD, "dK")
    check(dV, dVw.cpu(), F32, "dV")


@pytest.mark.parametrize("dq,dy,out", [("f32", "bf16", "f32"), ("bf16", "f32", "bf16"), ("bf16", "bf16", "f32"), ("f32", "f32", "bf16")])
def test_types_of_one_call_can_differ(fs, dq, dy, out):
    import torch
    types = {"f32": torch.float32, "bf16": torch.bfloat16}
    d, M, B, H, L = 64, 64, 3, 2, 150
    gen = torch.Generator().manual_seed(3)
    s = d ** -0.25
    theta, omega = make_theta(gen, "dense", H, d), torch.randn((H, M, d), generator=gen)
    o, f = oracle(theta, omega, s, H), fs.state_prepare(theta.cuda(), omega.cuda(), s)
    K, V = rows(gen, torch.float32, B, H, L, d), rows(gen, torch.float32, B, H, L, d)
    Q, dY = rows(gen, types[dq], B, H, L, d), rows(gen, types[dy], B, H, L, d)
    state = fs.state_append(f, fs.state_new(B, H, M, d), K, V)
    Y = fs.state_attention(f, state, Q, out_dtype=types[out])
    dQ, ds = fs.state_attention_backward(f, state, Q, dY, grad_dtype=types[out])
    assert Y.dtype == dQ.dtype == types[out]
    for b in range(B):
        for h in range(H):
            st = (state.T[b, h].double(), state.z[b, h].double(), None)
            check(Y[b, h], o.read(st, h, Q[b, h].double()).cpu(), F32, "Y")
            q, T, z = o.read_backward(st, h, Q[b, h].double(), dY[b, h].double())
            check(dQ[b, h], q.cpu(), GRAD, "dQ", parts_of(o, st, h, dY[b, h].double()).cpu())
            check(ds.T[b, h].reshape(1, -1), T.reshape(1, -1).cpu(), F32, "dT")
            check(ds.z[b, h][None], z[None].cpu(), GRAD, "dz")


@pytest.mark.parametrize("family", ["iso", "dense"])
def test_more_rows_than_a_grid_dimension(fs, family):
    """17 million keys (2^20 tiles of sixteen rows and some) and 4.3 million queries (2^15 pieces of 128 and some).  A sum that a workgroup takes
    alone has up to 8400 chunks, each addition of which is off by half a step: 8400 * 2^-24 = 5e-4."""
    import torch
    d, M, dt = 4, 32, torch.bfloat16
    L, LQ = (1 << 24) + 333, (1 << 22) + 777
    gen = torch.Generator().manual_seed(5)
    s = d ** -0.25
    theta, omega = make_theta(gen, family, 1, d), torch.randn((1, M, d), generator=gen)
    o, f = oracle(theta, omega, s, 1), fs.state_prepare(theta.cuda(), omega.cuda(), s)
    dev = torch.Generator(device="cuda").manual_seed(6)
    K, V = (torch.randn((1, 1, L, 8), generator=dev, device="cuda").to(dt)[..., :d] for _ in range(2))
    V += 1
    state = fs.state_append(f, fs.state_new(1, 1, M, d), K, V)
    st = (torch.zeros((M, d), dtype=torch.float64, device="cuda"), torch.zeros(M, dtype=torch.float64, device="cuda"),
          torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
    for i in range(0, L, 1 << 20):
        st = o.append(st, 0, 0, K[0, 0, i:i + (1 << 20)].double(), V[0, 0, i:i + (1 << 20)].double())
    assert abs(float(state.shift) - float(st[2])) <= 2e-5
    check(state.T[0, 0].reshape(1, -1), st[0].reshape(1, -1).cpu(), F32 + 5e-4, "T")
    check(state.z[0], st[1][None].cpu(), F32 + 5e-4, "z")
    Q = K[:, :, :LQ]
    Y = fs.state_attention(f, state, Q)
    own = (state.T[0, 0].double(), state.z[0, 0].double(), None)
    for i in (0, LQ - 5000, 1 << 22, (1 << 22) - 300):
        check(Y[0, 0, i:i + 500], o.read(own, 0, Q[0, 0, i:i + 500].double()).cpu(), F32, "Y")
    g = [torch.randn(t.shape, generator=gen).cuda() for t in state[:2]]
    dK, dV = fs.state_append_backward(f, state, fs.State(*g, None), Q, V[:, :, :LQ])
    for i in (0, LQ - 400, 1 << 22):
        k, v = o.append_backward(state.shift[0, 0].double(), 0, Q[0, 0, i:i + 300].double(), V[0, 0, i:i + 300].double(), g[0][0, 0].double(), g[1][0, 0].double())
        check(dK[0, 0, i:i + 300], k.cpu(), GRAD, "dK")
        check(dV[0, 0, i:i + 300], v.cpu(), F32, "dV")


@pytest.mark.parametrize("B,heads,G,d,M", [(70, 4, 1, 64, 256), (3, 2, 4, 128, 512), (2, 2, 1, 64, 288), (64, 4, 1, 64, 256), (2, 1, 3, 40, 2048)])
def test_two_graphs_share_a_workspace(fs, B, heads, G, d, M):
    """Tokens in one launch and in two, and an append, captured twice with the same workspace and replayed in turn."""
    import torch
    gen = torch.Generator().manual_seed(B)
    s, dt, L = d ** -0.25, torch.bfloat16, 90
    theta, omega = make_theta(gen, "dense", heads, d).cuda(), torch.randn((heads, M, d), generator=gen).cuda()
    f, rot = fs.state_prepare(theta, omega, s), fs.Rotary(fs.rotary_frequencies(d), None)
    ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    K, V, q, k, v = (rows(gen, dt, B, h, n, d) for h, n in ((heads, L), (heads, L), (heads * G, 1), (heads, 1), (heads, 1)))
    states = [fs.state_new(B, heads, M, d) for _ in range(3)]
    def work(state, scale):
        fs.state_append(f, state, K * scale, V, rotary=rot, fresh=True, workspace=ws)
        return fs.state_step(f, state, q, k * scale, v, rotary=rot, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(states[0], 1.0)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            outs.append(work(states[i], 1.0 - 0.5 * i))
    for turn in range(3):
        for t in (K, V, q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen).to(dt))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [[outs[i].clone(), *(t.clone() for t in states[i])] for i in range(2)]
        for i in range(2):
            want = [work(states[2], 1.0 - 0.5 * i), *states[2]]
            assert all(torch.equal(x, y) for x, y in zip(got[i], want)), (turn, i)


@pytest.mark.parametrize("B,heads,G,d,dv,M,family", [(300, 1, 1, 64, 64, 256, "iso"), (40, 7, 1, 32, 30, 64, "dense"), (3, 1, 4, 128, 128, 1024, "dense"),
                                                   (17, 2, 5, 64, 64, 96, "iso"), (2, 1, 1, 64, 64, 2048, "iso"), (5, 3, 1, 20, 48, 256, "dense")])
def test_steps_in_one_launch_and_two(fs, B, heads, G, d, dv, M, family):
    """Tokens onto states with rows, with a sequence that has none and one that shares its state, against append and attention in 64 bits."""
    import torch
    gen = torch.Generator().manual_seed(B + M)
    s, L = d ** -0.25, 40
    theta, omega = make_theta(gen, family, heads, d), torch.randn((heads, M, d), generator=gen)
    o, f = oracle(theta, omega, s, heads), fs.state_prepare(theta.cuda(), omega.cuda(), s)
    K, V = rows(gen, torch.float32, B, heads, L, d), rows(gen, torch.float32, B, heads, L, dv)
    q, k, v = (rows(gen, torch.float32, B, *n) for n in ((heads * G, 1, d), (heads, 1, d), (heads, 1, dv)))
    slots = torch.randperm(B, generator=gen).to(torch.int32)
    state = fs.state_append(f, fs.state_new(B, heads, M, dv), K, V)
    before = [t.clone() for t in state]
    if B > 2:
        slots[1], slots[2] = -1, slots[0]
    unread = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = fs.state_step(f, state, q, k, v, slots=slots.cuda(), unread=unread)
    out = [1, 2] if B > 2 else []
    assert int(unread) == len(out) * heads * G
    used = {int(x) for i, x in enumerate(slots) if i not in out}
    for i in range(B):
        if i not in used:
            assert all(torch.equal(a[i], b[i]) for a, b in zip(before, state))
    for i in range(B):
        for h in range(heads):
            if i in out:
                assert (Y[i, h * G:(h + 1) * G] == 0).all()
                continue
            slot = int(slots[i])
            st = o.append(tuple(t[slot, h].double() for t in before), i, h, k[i, h].double(), v[i, h].double())
            scale = torch.exp2(st[2] - state.shift[slot, h].double())
            assert abs(float(scale) - 1) <= 2e-5
            check(state.T[slot, h].reshape(1, -1), (st[0] * scale).reshape(1, -1).cpu(), F32, "T")
            check(state.z[slot, h][None], (st[1] * scale)[None].cpu(), F32, "z")
            for g in range(G):
                check(Y[i, h * G + g], o.read(st, h, q[i, h * G + g].double()).cpu(), F32, "Y")
