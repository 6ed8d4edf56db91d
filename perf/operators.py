"""Rotary positions and attention through kept states, as measurable cases.

With positive random features the keys and values of a sequence enter attention only through a state per key head: with the
exponents (base 2) of the key features

    e[j, m] = (W2 k_j)_m + bias_m + r(k_j),   W2 = log2(e) s Omega B2,   bias_m = log2(e) (w_m' A w_m + log D - log(M) / 2),
    r(k) = log2(e) s^2 k' C2 k,

a state is shift = max e, z_m = sum_j 2^(e[j, m] - shift), T_m = sum_j 2^(e[j, m] - shift) V_j (nothing appended: shift = -inf,
T = z = 0), and a query reads it as y = sum_m p_m T_m / sum_m p_m z_m, p_m = 2^((W1 q)_m + bias_m), W1 = log2(e) s Omega B1;
zero where the state is empty.  The cases:

  rotary   queries and keys turned by their positions in one call (backward: turned back)
  append   the keys and values of a padded batch, turned on the way, into the states that a pool keeps
  read     attention of queries to states of the pool (cross attention to an encoder, or a prompt's next part)
  train    cross attention to a padded encoder batch, forward and backward
  step     one token of every sequence: appended, then read
"""
from __future__ import annotations

import math

import torch

own = False

LOG2E = 1.0 / math.log(2.0)


def _rotary(dtype, B, H, Hk, L, d, rot, interleaved, scaling, transposed):
    return dict(op="rotary", dtype=dtype, B=B, H=H, Hk=Hk, L=L, d=d, rot=rot, interleaved=interleaved, scaling=scaling,
                transposed=transposed)


def _append(dtype, B, Hk, L, d, dv, M, rot, family, fresh):
    return dict(op="append", dtype=dtype, B=B, Hk=Hk, L=L, d=d, dv=dv, M=M, rot=rot, family=family, fresh=fresh)


def _read(dtype, B, H, Hk, L, d, dv, M, rot, family):
    return dict(op="read", dtype=dtype, B=B, H=H, Hk=Hk, L=L, d=d, dv=dv, M=M, rot=rot, family=family)


def _train(dtype, B, H, Hk, L, Lk, d, dv, M, family):
    return dict(op="train", dtype=dtype, B=B, H=H, Hk=Hk, L=L, Lk=Lk, d=d, dv=dv, M=M, rot=0, family=family)


def _step(dtype, B, H, Hk, d, dv, M, rot, family):
    return dict(op="step", dtype=dtype, B=B, H=H, Hk=Hk, L=1, d=d, dv=dv, M=M, rot=rot, family=family)


def listed():
    cases = [
        # the new token of 32 sequences: what a decoder does between two launches, all latency
        ("rotary_token", _rotary("bf16", 32, 8, 8, 1, 64, 64, False, "plain", False)),
        # queries and keys of a training step on the headline shapes, frequencies scaled for a long context
        ("rotary_train", _rotary("bf16", 4, 8, 8, 16384, 64, 64, False, "blend", False)),
        # gradients turned back: fp32, interleaved pairs, part of the head, shared key heads, an odd length
        ("rotary_back", _rotary("f32", 3, 12, 4, 1777, 128, 96, True, "linear", True)),
        # prompts of different lengths of a serving batch, into new states
        ("prompt_append", _append("bf16", 8, 8, 4096, 64, 64, 256, 64, "iso", True)),
        # the next part of a few documents onto the states that they have, fp32, dense quadratic forms
        ("chunk_append", _append("f32", 5, 3, 77, 32, 32, 512, 16, "dense", False)),
        # decoder queries of a batch on the encoder states that it keeps, two query heads to a key head
        ("encoder_read", _read("bf16", 8, 16, 8, 2048, 64, 64, 256, 0, "iso")),
        # one short fp32 sequence: launches and host time
        ("small_read", _read("f32", 1, 1, 1, 256, 16, 16, 64, 0, "iso")),
        # the cross attention of a training step, encoder batch padded
        ("cross_train", _train("bf16", 8, 8, 8, 1024, 4096, 64, 64, 256, "iso")),
        # the same on wide heads in fp32, dense quadratic forms, two query heads to a key head, odd lengths
        ("cross_train_wide", _train("f32", 1, 8, 4, 501, 1499, 128, 128, 512, "dense")),
        # the next token of one sequence
        ("token_one", _step("bf16", 1, 8, 8, 64, 64, 256, 64, "iso")),
        # the next token of a full serving batch
        ("token_batch", _step("bf16", 256, 8, 8, 64, 64, 256, 64, "iso")),
        # wide heads, four query heads to a key head, an odd batch
        ("token_shared", _step("bf16", 45, 16, 4, 128, 128, 512, 128, "dense")),
    ]
    return [dict(name=name, **case) for name, case in cases]


# ------------------------------------------------------------------------------------------------ drawn cases
def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "append", "append", "read", "read", "train", "train", "step", "step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    family = rng.choice(["iso", "iso", "dense"])
    Hk = rng.choice([1, 2, 3, 4, 8])
    H = Hk * rng.choice([1, 1, 2, 3, 4])
    d = rng.choice([16, 24, 32, 48, 64, 64, 80, 96, 128])
    dv = rng.choice([d, d, d, 40, 64, 128])
    M = rng.choice([32, 64, 100, 128, 200, 256, 256, 384, 512])
    rot = rng.choice([0, d, d, d // 2])
    wide = max(1, d * M // 16384)
    if op == "rotary":
        rows = _log_uniform(rng, 8, 1 << 19)
        L = _log_uniform(rng, 1, max(1, min(16384, rows // H)))
        return _rotary(dtype, max(1, rows // (H * L)), H, Hk, L, d, rot or d, rng.random() < 0.5,
                       rng.choice(["plain", "linear", "base", "blend"]), rng.random() < 0.4)
    if op == "append":
        rows = _log_uniform(rng, 16, (1 << 17) // wide)
        L = _log_uniform(rng, 1, max(1, min(8192, rows // Hk)))
        return _append(dtype, max(1, rows // (Hk * L)), Hk, L, d, dv, M, rot, family, rng.random() < 0.5)
    if op == "read":
        rows = _log_uniform(rng, 16, (1 << 17) // wide)
        L = _log_uniform(rng, 1, max(1, min(4096, rows // H)))
        return _read(dtype, min(64, max(1, rows // (H * L))), H, Hk, L, d, dv, M, rot, family)
    if op == "train":
        rows = _log_uniform(rng, 64, (1 << 16) // wide)
        L = _log_uniform(rng, 8, max(8, min(2048, rows // H)))
        return _train(dtype, min(64, max(1, rows // (H * L))), H, Hk, L, min(_log_uniform(rng, 16, 4096), 8 * L), d, dv, M, family)
    return _step(dtype, max(1, _log_uniform(rng, 1, 512) // wide), H, Hk, d, dv, M, rot, family)


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _frequencies(rot, scaling):
    """Radians a position for each pair, and the factor of the turned values."""
    i = torch.arange(0, rot, 2, dtype=torch.float64) / rot
    f = 10000.0 ** -i
    if scaling == "linear":
        return f / 4.0, 1.0
    if scaling == "base":
        return (10000.0 * 4.0 ** (rot / max(rot - 2.0, 1.0))) ** -i, 1.0
    if scaling == "blend":         # pairs of long wavelengths stretched, short ones kept, a ramp between
        turns = 4096.0 * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        return f * keep + f / 4.0 * (1.0 - keep), 0.1 * math.log(4.0) + 1.0
    return f, 1.0


def _theta(gen, family, groups, d):
    """Parameter sets as the library lays them out: A = a I, B1 = b G, B2 = b G^-T, C1 = -G'G / 2, C2 = -G^-1 G^-T / 2."""
    a = -0.02 - 0.06 * torch.rand((groups,), generator=gen, device="cuda", dtype=torch.float64)
    b, eye = torch.sqrt(1.0 - 4.0 * a)[:, None, None], torch.eye(d, dtype=torch.float64, device="cuda").expand(groups, d, d)
    G, inv = eye, eye
    if family == "dense":
        N = torch.randn((groups, d, d), generator=gen, device="cuda", dtype=torch.float64) * (0.15 / math.sqrt(d))
        G = eye + N
        inv = torch.linalg.inv(G)
    head = torch.zeros((groups, 8), dtype=torch.float64, device="cuda")
    head[:, 0] = 0.25 * d * torch.log(1.0 - 4.0 * a)
    head[:, 1] = math.nan
    head[:, 2] = 3.0 if family == "iso" else 0.0
    head[:, 3] = 1.0 if family == "iso" else 3.0
    parts = [head, a[:, None].expand(groups, d), b * G, b * inv.transpose(1, 2), -0.5 * G.transpose(1, 2) @ G,
             -0.5 * inv @ inv.transpose(1, 2)]
    return torch.cat([p.reshape(groups, -1) for p in parts], dim=1).float().contiguous()


def _constants(theta, omega, s, dt):
    """W1, W2, bias, C2 of every parameter set in dt, from the fp32 parameters."""
    g, M, d = omega.shape
    th, om = theta.to(dt), omega.to(dt)
    A, B1, B2, _, C2 = (th[:, 8 + a:8 + b] for a, b in ((0, d), (d, d + d * d), (d + d * d, d + 2 * d * d),
                                                          (d + 2 * d * d, d + 3 * d * d), (d + 3 * d * d, d + 4 * d * d)))
    bias = LOG2E * ((om * om * A[:, None, :]).sum(-1) + th[:, :1] - 0.5 * math.log(M))
    return LOG2E * s * (om @ B1.reshape(g, d, d)), LOG2E * s * (om @ B2.reshape(g, d, d)), bias, C2.reshape(g, d, d)


def _rows(gen, B, H, L, d, s, dt):
    x = torch.randn((B, H, L, d), generator=gen, device="cuda")
    m = torch.randn((H, 1, d), generator=gen, device="cuda")
    return (x + 0.5 / s * m / m.norm(dim=-1, keepdim=True)).to(dt)


def _lengths(gen, B, L):
    """Lengths of a padded batch: the first sequence fills it, the others hold a half and more of it or, one in eight, little."""
    u = torch.rand((B,), generator=gen, device="cuda")
    few = torch.rand((B,), generator=gen, device="cuda") < 0.125
    n = torch.where(few, u * 0.1, 0.5 + 0.5 * u) * L
    n[0] = L
    return n.round().clamp(1, L).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dt, B, d = case["op"], _dtype(case), case["B"], case["d"]
    Hk, s = case["Hk"], float(case["d"]) ** -0.25
    st = dict(case=case, s=s)
    if case["rot"]:
        # documents and conversations of any age: a first position of each, then one after the other
        freqs, st["amplitude"] = _frequencies(case["rot"], case.get("scaling", "plain"))
        st["freqs"] = freqs.cuda()
        first = torch.randint(0, 100000, (B, 1), generator=gen, device="cuda")
        st["positions"] = (first + torch.arange(case["L"], device="cuda")).to(torch.int32)
    if op == "rotary":
        st["Q"], st["K"] = (_rows(gen, B, h, case["L"], d, s, dt) for h in (case["H"], Hk))
        return st
    M, dv = case["M"], case["dv"]
    theta = _theta(gen, case["family"], Hk, d)
    omega = torch.randn((Hk, M, d), generator=gen, device="cuda")
    st["theta"], st["omega"] = theta, omega
    # the projection constants of the parameters, kept while those stay
    st["W1"], st["W2"], st["bias"], st["C2"] = (t.float() for t in _constants(theta, omega, s, torch.float64))
    if own:
        from paper_2302_00787_amd import binding as fs
        st["features"] = fs.state_prepare(theta, omega, s)
    if op == "train":
        st["K"] = _rows(gen, B, Hk, case["Lk"], d, s, dt)
        st["V"] = torch.randn((B, Hk, case["Lk"], dv), generator=gen, device="cuda").to(dt)
        st["lengths"] = _lengths(gen, B, case["Lk"])
        st["Q"] = _rows(gen, B, case["H"], case["L"], d, s, dt)
        st["dY"] = torch.randn((B, case["H"], case["L"], dv), generator=gen, device="cuda").to(dt)
        return st
    # a pool with states to spare, the batch's in any order; the states of texts of 24 tokens
    n = B + 3
    st["slots"] = torch.randperm(n, generator=gen, device="cuda")[:B].to(torch.int32)
    k = _rows(gen, n, Hk, 24, d, s, torch.float32)
    e = k @ st["W2"].transpose(1, 2) + st["bias"][:, None, :] + LOG2E * s * s * ((k @ st["C2"]) * k).sum(-1, keepdim=True)
    st["shift"] = e.amax(dim=(2, 3)).contiguous()
    S = torch.exp2(e - st["shift"][..., None, None])
    st["z"] = S.sum(2).contiguous()
    st["T"] = (S.transpose(2, 3) @ torch.randn((n, Hk, 24, dv), generator=gen, device="cuda")).contiguous()
    if op in ("append", "step"):
        st["K"] = _rows(gen, B, Hk, case["L"], d, s, dt)
        st["V"] = torch.randn((B, Hk, case["L"], dv), generator=gen, device="cuda").to(dt)
    if op == "append":
        st["lengths"] = _lengths(gen, B, case["L"])
    if op in ("read", "step"):
        st["Q"] = _rows(gen, B, case["H"], case["L"], d, s, dt)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def _own(st):
    from paper_2302_00787_amd import binding as fs
    case = st["case"]
    op = case["op"]
    rot = None
    if case["rot"]:
        rot = fs.Rotary(st["freqs"], st["positions"], case.get("interleaved", False), st["amplitude"])
    if op == "rotary":
        return fs.rotary(st["Q"], rot, st["K"], transposed=case["transposed"])
    f = st["features"]
    if op == "train":
        state = fs.state_new(case["B"], case["Hk"], case["M"], case["dv"], device=st["K"].device)
        fs.state_append(f, state, st["K"], st["V"], lengths=st["lengths"], fresh=True)
        Y = fs.state_attention(f, state, st["Q"])
        dQ, dstate = fs.state_attention_backward(f, state, st["Q"], st["dY"])
        dK, dV = fs.state_append_backward(f, state, dstate, st["K"], st["V"], lengths=st["lengths"])
        return Y, dQ, dK, dV
    state = fs.State(st["T"], st["z"], st["shift"])
    if op == "append":
        fs.state_append(f, state, st["K"], st["V"], lengths=st["lengths"], slots=st["slots"], rotary=rot, fresh=case["fresh"])
        return tuple(state)
    if op == "read":
        return fs.state_attention(f, state, st["Q"], slots=st["slots"], rotary=rot)
    Y = fs.state_step(f, state, st["Q"], st["K"], st["V"], slots=st["slots"], rotary=rot)
    return (Y,) + tuple(state)


def _turned(x, st, transposed=False):
    """Rows [B, H, L, d] in 32 bits turned by their positions, the angles in 64."""
    case, r = st["case"], st["case"]["rot"] // 2
    if not r:
        return x
    angle = st["positions"].double()[:, None, :, None] * st["freqs"]
    c, s = (st["amplitude"] * torch.cos(angle)).float(), (st["amplitude"] * torch.sin(angle)).float()
    if transposed:
        s = -s
    if case.get("interleaved", False):
        u, v = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
        turned = torch.stack([u * c - v * s, v * c + u * s], dim=-1).flatten(-2)
    else:
        u, v = x[..., :r], x[..., r:2 * r]
        turned = torch.cat([u * c - v * s, v * c + u * s], dim=-1)
    return torch.cat([turned, x[..., 2 * r:]], dim=-1)


def _key_exponents(st, k):
    """[B, Hk, L, M] from turned keys."""
    r = ((k @ st["C2"]) * k).sum(-1, keepdim=True) * (LOG2E * st["s"] ** 2)
    return k @ st["W2"].transpose(1, 2) + st["bias"][:, None, :] + r


def _query_features(st, q):
    """[B, Hk, query heads of a key head times L, M], every row on its own maximum."""
    case = st["case"]
    q = q.reshape(case["B"], case["Hk"], -1, case["d"])
    e = q @ st["W1"].transpose(1, 2) + st["bias"][:, None, :]
    return torch.exp2(e - e.amax(-1, keepdim=True))


def _behind(lengths, L):
    return torch.arange(L, device="cuda") >= lengths[:, None]


def _quotient(num, den):
    return torch.where(den > 0, num / den, torch.zeros_like(num))


def _appended(st, k, V, lengths, T, z, shift):
    """State after keys (turned) and values, from the one before."""
    behind = _behind(lengths, k.shape[2])[:, None, :, None]
    e = _key_exponents(st, k).masked_fill(behind, -math.inf)
    new = torch.maximum(shift, e.amax(dim=(2, 3)))
    S = torch.exp2(e - new[..., None, None])
    keep = torch.exp2(shift - new)[..., None]
    return T * keep[..., None] + S.transpose(2, 3) @ V.masked_fill(behind, 0.0), z * keep + S.sum(2), new


def run(st):
    if own:
        return _own(st)
    case = st["case"]
    op, dt = case["op"], _dtype(case)
    if op == "rotary":
        return tuple(_turned(st[x].float(), st, case["transposed"]).to(dt) for x in ("Q", "K"))
    if op == "train":
        return _train_plain(st)
    T, z, shift, at = st["T"], st["z"], st["shift"], st["slots"].long()
    if op in ("append", "step"):
        old = (T[at], z[at], shift[at])
        if case.get("fresh", False):
            old = tuple(torch.full_like(t, f) for t, f in zip(old, (0.0, 0.0, -math.inf)))
        n = st["lengths"] if op == "append" else torch.ones_like(st["slots"])
        T[at], z[at], shift[at] = _appended(st, _turned(st["K"].float(), st), st["V"].float(), n, *old)
        if op == "append":
            return T, z, shift
    p = _query_features(st, _turned(st["Q"].float(), st))
    Y = _quotient(p @ T[at], (p * z[at][:, :, None, :]).sum(-1, keepdim=True))
    Y = Y.reshape(case["B"], case["H"], case["L"], case["dv"]).to(dt)
    return Y if op == "read" else (Y, T, z, shift)


def _train_plain(st):
    case, dt = st["case"], _dtype(st["case"])
    B, H, Hk, L, Lk, d, dv = (case[x] for x in ("B", "H", "Hk", "L", "Lk", "d", "dv"))
    k, v = st["K"].float(), st["V"].float()
    behind = _behind(st["lengths"], Lk)[:, None, :, None]
    e = _key_exponents(st, k).masked_fill(behind, -math.inf)
    S = torch.exp2(e - e.amax(dim=(2, 3), keepdim=True))
    T, z = S.transpose(2, 3) @ v, S.sum(2)[:, :, None, :]
    p = _query_features(st, st["Q"].float())
    den = (p * z).sum(-1, keepdim=True)
    Y = _quotient(p @ T, den)
    p = _quotient(p, den)
    dY = st["dY"].float().reshape(B, Hk, -1, dv)
    delta = (dY * Y).sum(-1, keepdim=True)
    dQ = ((p * (dY @ T.transpose(2, 3) - delta * z)) @ st["W1"]) / LOG2E
    dT, dz = p.transpose(2, 3) @ dY, -(p * delta).sum(2)[:, :, None, :]
    dE = S * (v @ dT.transpose(2, 3) + dz)
    C = st["C2"] + st["C2"].transpose(1, 2)
    dK = (dE @ st["W2"]) / LOG2E + dE.sum(-1, keepdim=True) * st["s"] ** 2 * (k @ C)
    return (Y.reshape(B, H, L, dv).to(dt), dQ.reshape(B, H, L, d).to(dt), dK.to(dt), (S @ dT).to(dt))


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    if case["op"] != "rotary" and case["B"] * case["M"] * (case["H"] * case["L"] if "H" in case else 0) > 1 << 30:
        return None
    st = prepare(case, seed)
    op, s = case["op"], st["s"]

    def turn(x):
        if not case["rot"]:
            return x
        n, y = case["rot"], x.clone()
        phase = torch.einsum("bl,i->bli", st["positions"].double(), st["freqs"]).unsqueeze(1)
        if case.get("transposed", False):
            phase = -phase
        pairs = y[..., :n].unflatten(-1, (n // 2, 2)) if case.get("interleaved", False) else y[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2)
        w = torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * torch.polar(torch.full_like(phase, st["amplitude"]), phase)
        out = torch.view_as_real(w)
        y[..., :n] = (out if case.get("interleaved", False) else out.transpose(-1, -2)).flatten(-2)
        return y

    if op == "rotary":
        return turn(st["Q"].double()), turn(st["K"].double())
    B, Hk, M = case["B"], case["Hk"], case["M"]
    th, om, d = st["theta"].double(), st["omega"].double(), case["d"]

    def block(i):
        return th[:, 8 + d + i * d * d:8 + d + (i + 1) * d * d].reshape(Hk, d, d)

    quad = (om.square() * th[:, None, 8:8 + d]).sum(-1) + th[:, :1] - 0.5 * math.log(M)           # natural logarithms here

    def log_key(b, h):
        y = s * k[b, h, :n[b]]
        return y @ block(1)[h].T @ om[h].T + quad[h] + (y * (y @ block(3)[h].T)).sum(1, keepdim=True)

    # sequence by sequence and head by head
    if op == "read":
        T, z, shift = (st[x].double() for x in ("T", "z", "shift"))
        at = st["slots"].tolist()
    else:
        n = st["lengths"].tolist() if op != "step" else [1] * B
        k, v = turn(st["K"].double()), st["V"].double()
        at = list(range(B)) if op == "train" else st["slots"].tolist()
        if op == "train":
            T = torch.zeros((B, Hk, M, case["dv"]), dtype=torch.float64, device="cuda")
            z, shift = T[..., 0].clone(), torch.full((B, Hk), -math.inf, dtype=torch.float64, device="cuda")
        else:
            T, z, shift = (st[x].double() for x in ("T", "z", "shift"))
        for b, a in enumerate(at):
            for h in range(Hk):
                if case.get("fresh", op == "train"):
                    T[a, h], z[a, h], shift[a, h] = 0.0, 0.0, -math.inf
                g = log_key(b, h)
                top = torch.maximum(shift[a, h], g.max() * LOG2E)
                f, old = torch.exp(g - top / LOG2E), torch.exp((shift[a, h] - top) / LOG2E)
                T[a, h] = T[a, h] * old + f.T @ v[b, h, :n[b]]
                z[a, h] = z[a, h] * old + f.sum(0)
                shift[a, h] = top
        if op == "append":
            return T, z, shift
    q = turn(st["Q"].double())
    H, G = case["H"], case["H"] // Hk
    Y = torch.empty((B, H, case["L"], case["dv"]), dtype=torch.float64, device="cuda")
    if op == "train":
        dQ, dK, dV = (torch.zeros_like(x) for x in (q, k, v))
        dY = st["dY"].double()
    for b, a in enumerate(at):
        for h in range(Hk):
            if op == "train":
                S = torch.exp(log_key(b, h) - shift[a, h] / LOG2E)
                dT, dz = torch.zeros_like(T[a, h]), torch.zeros_like(z[a, h])
            for i in range(h * G, (h + 1) * G):
                g = s * q[b, i] @ block(0)[h].T @ om[h].T + quad[h]
                P = torch.exp(g - g.max(1, keepdim=True).values)
                P = P / (P @ z[a, h])[:, None]
                Y[b, i] = P @ T[a, h]
                if op == "train":
                    delta = (dY[b, i] * Y[b, i]).sum(1)
                    dT += P.T @ dY[b, i]
                    dz -= P.T @ delta
                    dQ[b, i] = s * (P * (dY[b, i] @ T[a, h].T - delta[:, None] * z[a, h])) @ om[h] @ block(0)[h]
            if op == "train":
                y = k[b, h, :n[b]]
                dV[b, h, :n[b]] = S @ dT
                dg = S * (v[b, h, :n[b]] @ dT.T + dz)
                dK[b, h, :n[b]] = s * dg @ om[h] @ block(1)[h] + s * s * dg.sum(1, keepdim=True) * (y @ (block(3)[h] + block(3)[h].T))
    if op == "train":
        return Y, dQ, dK, dV
    return Y if op == "read" else (Y, T, z, shift)


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    """Inputs read once and outputs written once; multiply-adds of the method (two flops each)."""
    op, B, d, Hk = case["op"], case["B"], case["d"], case["Hk"]
    size = 2 if case["dtype"] == "bf16" else 4
    turns = 4 * B * case["L"] if case["rot"] else 0
    if op == "rotary":
        rows = B * case["L"] * (case["H"] + Hk)
        return {"bytes": 2 * rows * d * size + turns, "flops": 3 * rows * case["rot"]}
    M, dv = case["M"], case["dv"]
    constants = 4 * Hk * M * (d + 1)
    state = 4 * B * Hk * (M * (dv + 1) + 1)
    contraction = 2 * M * (d + dv + 1)         # of one row: its features and their products with a state
    if op == "append":
        rows = B * Hk * case["L"] * 3 // 4     # a quarter of the batch is padding
        return {"bytes": rows * (d + dv) * size + state * (1 if case["fresh"] else 2) + constants + turns, "flops": rows * contraction}
    rows = B * case["H"] * case["L"]
    if op == "read":
        return {"bytes": rows * (d + dv) * size + state + constants + turns, "flops": rows * contraction}
    if op == "step":
        keys = B * Hk
        return {"bytes": (rows + keys) * (d + dv) * size + 2 * state + 2 * constants + turns, "flops": (rows + keys) * contraction}
    keys = B * Hk * case["Lk"] * 3 // 4
    # forward: features and states, features and outputs.  Backward: each side's features and products with a state again, and of each
    # product one with respect to its other factor
    return {"bytes": (rows * (2 * d + 2 * dv) + keys * (2 * d + 2 * dv)) * size + 2 * constants,
            "flops": rows * (contraction + 4 * d * M + 4 * M * (dv + 1)) + keys * (contraction + 4 * d * M + 4 * M * (dv + 1))}
