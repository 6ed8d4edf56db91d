"""Linear attention with a decay for each head, and rotary positions with several axes, as measurable cases.

A state S [d, dv] of a sequence and a key head forgets: with lambda = exp(g) <= 1, g the head's log decay,

    S_i = lambda S_(i-1) + k_i v_i',   y_i = scale q_i S_i,                                S_(-1) = S before the call (or zero),

which over the rows of a call is y_i = scale (lambda^(i+1) q_i S_before + sum_(j <= i) lambda^(i-j) (q_i . k_j) v_j).  H query heads share
Hk key heads, their decays and their states.  Gradients of sum(Y * dY) + sum(S_after * dS_after), with
D_j = lambda^(n-1-j) dS_after + scale sum_(i >= j) lambda^(i-j) q_i dy_i':

    dq_i = scale S_i dy_i,   dk_j = D_j v_j,   dv_j = D_j' k_j,   dS_before = lambda D_0.

A position with several axes (time, height, width) has a number for each; pair p of a row belongs to one axis and is turned by the
angle position[axis of p] freqs[p].  The cases:

  prompt   the rows of a padded batch after what the states of a pool hold; the states go on
  train    forward and backward; with states before and after that have gradients, or one that all sequences begin with
  token    one token of every sequence, its state in place
  turn     queries and keys turned by positions with several axes in one call (backward: turned back)
"""
from __future__ import annotations

import math

import torch

own = False


def _prompt(dtype, B, H, Hk, L, d, dv, decay, fresh):
    return dict(op="prompt", dtype=dtype, B=B, H=H, Hk=Hk, L=L, d=d, dv=dv, decay=decay, fresh=fresh)


def _train(dtype, B, H, Hk, L, d, dv, decay, initial):
    return dict(op="train", dtype=dtype, B=B, H=H, Hk=Hk, L=L, d=d, dv=dv, decay=decay, initial=initial)


def _token(dtype, B, H, Hk, d, dv, decay):
    return dict(op="token", dtype=dtype, B=B, H=H, Hk=Hk, L=1, d=d, dv=dv, decay=decay)


def _turn(dtype, B, H, Hk, L, d, rot, axes, order, interleaved, transposed):
    return dict(op="turn", dtype=dtype, B=B, H=H, Hk=Hk, L=L, d=d, rot=rot, axes=axes, order=order, interleaved=interleaved,
                transposed=transposed)


def listed():
    cases = [
        # one short fp32 prompt into a new state: launches and host time
        ("prompt_short", _prompt("f32", 1, 2, 2, 77, 32, 32, "slow", True)),
        # the next part of the prompts of a serving batch, of different lengths, after what their states hold
        ("prompt_batch", _prompt("bf16", 8, 8, 8, 4096, 64, 64, "slow", False)),
        # one long document on wide heads
        ("prompt_long", _prompt("bf16", 1, 16, 16, 65536, 128, 128, "slow", True)),
        # a training step on long sequences
        ("train", _train("bf16", 4, 8, 8, 16384, 64, 64, "slow", "none")),
        # parts of documents whose states go from step to step with their gradients, fp32, shared key heads, odd sizes
        ("train_carried", _train("f32", 3, 12, 4, 1777, 96, 128, "steep", "own")),
        # many short texts that begin with one learned state
        ("train_texts", _train("bf16", 64, 8, 8, 1024, 64, 64, "slow", "shared")),
        # the next token of one sequence
        ("token_one", _token("bf16", 1, 8, 8, 64, 64, "slow")),
        # the next token of a full serving batch
        ("token_batch", _token("bf16", 256, 8, 8, 64, 64, "slow")),
        # fp32, wide heads, four query heads to a key head, an odd batch
        ("token_shared", _token("f32", 45, 16, 4, 128, 128, "steep")),
        # the new tokens of 32 sequences, between two launches of a decoder
        ("turn_token", _turn("bf16", 32, 8, 8, 1, 64, 64, 3, "blocks", False, False)),
        # a training step on clips of 16 frames of 32 x 32 patches
        ("turn_video", _turn("bf16", 4, 8, 8, 16384, 64, 64, 3, "cyclic", False, False)),
        # gradients turned back: images, fp32, interleaved pairs, part of the head, shared key heads, an odd length
        ("turn_back", _turn("f32", 3, 12, 4, 1777, 128, 96, 2, "blocks", True, True)),
    ]
    return [dict(name=name, **case) for name, case in cases]


# ------------------------------------------------------------------------------------------------ drawn cases
def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "train", "train", "token", "turn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    decay = rng.choice(["slow", "slow", "steep", "none"])
    Hk = rng.choice([1, 2, 3, 4, 8])
    H = Hk * rng.choice([1, 1, 2, 3, 4])
    d = rng.choice([16, 24, 32, 48, 64, 64, 80, 96, 128])
    dv = rng.choice([d, d, d, 40, 64, 128])
    wide = max(1, max(d, dv) // 64) * (2 if dtype == "f32" else 1)
    if op == "turn":
        rows = _log_uniform(rng, 8, 1 << 19)
        L = _log_uniform(rng, 1, max(1, min(16384, rows // H)))
        rot = rng.choice([d, d, d // 2])
        return _turn(dtype, max(1, rows // (H * L)), H, Hk, L, d, rot, rng.choice([2, 3, 3]), rng.choice(["blocks", "cyclic"]),
                     rng.random() < 0.5, rng.random() < 0.4)
    if op == "prompt":
        rows = _log_uniform(rng, 16, (1 << 19) // wide)
        L = _log_uniform(rng, 1, max(1, min(16384, rows // H)))
        return _prompt(dtype, min(256, max(1, rows // (H * L))), H, Hk, L, d, dv, decay, rng.random() < 0.5)
    if op == "train":
        rows = _log_uniform(rng, 64, (1 << 18) // wide)
        L = _log_uniform(rng, 2, max(2, min(8192, rows // H)))
        return _train(dtype, min(256, max(1, rows // (H * L))), H, Hk, L, d, dv, decay, rng.choice(["none", "none", "own", "shared"]))
    return _token(dtype, max(1, _log_uniform(rng, 1, 512) // wide), H, Hk, d, dv, decay)


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _log_decay(gen, decay, heads):
    """Heads that remember from 2^5 to 2^12 tokens, from 1 to 2^8, or everything."""
    if decay == "none":
        return torch.zeros((heads,), device="cuda")
    u = (torch.arange(heads, device="cuda") + torch.rand((heads,), generator=gen, device="cuda")) / heads
    return -torch.exp2(-5.0 - 7.0 * u) if decay == "slow" else -torch.exp2(-8.0 * u)


def _lengths(gen, B, L):
    """Lengths of a padded batch: the first sequence fills it, the others hold a half and more of it or, one in eight, little."""
    u = torch.rand((B,), generator=gen, device="cuda")
    few = torch.rand((B,), generator=gen, device="cuda") < 0.125
    n = torch.where(few, u * 0.1, 0.5 + 0.5 * u) * L
    n[0] = L
    return n.round().clamp(1, L).to(torch.int32)


def _grid_positions(gen, axes, B, L):
    """[axes, B, L]: clips (or images) of rows of up to 32 patches after a text of any length, whose axes go on together."""
    width = 1 + torch.randint(1, 32, (B, 1), generator=gen, device="cuda")
    height = 1 + torch.randint(1, 32, (B, 1), generator=gen, device="cuda")
    first = torch.randint(0, 100000, (B, 1), generator=gen, device="cuda")
    l = torch.arange(L, device="cuda")[None]
    places = [first + l // (width * height), first + l // width % height, first + l % width]
    return torch.stack(places[3 - axes:]).to(torch.int32)


def _sections(rot, axes, order):
    """Radians a position and axis of each pair: the axes share the pairs evenly, the first has the rest; in blocks, each with
    frequencies of its own, or in turn, with those of the whole row."""
    pairs = rot // 2
    n = [pairs // axes] * axes
    n[0] += pairs - sum(n)
    if order == "blocks":
        f = torch.cat([10000.0 ** -(torch.arange(m, dtype=torch.float64) / m) for m in n])
        return f, torch.cat([torch.full((m,), a, dtype=torch.int32) for a, m in enumerate(n)])
    return 10000.0 ** -(torch.arange(pairs, dtype=torch.float64) / pairs), (torch.arange(pairs) % axes).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dt, B, H, Hk, L, d = (case[x] for x in ("op", "dtype", "B", "H", "Hk", "L", "d"))
    dt = _dtype(case)

    def rows(heads, width):
        return torch.randn((B, heads, L, width), generator=gen, device="cuda").to(dt)

    st = dict(case=case, Q=rows(H, d), K=rows(Hk, d))
    if op == "turn":
        f, a = _sections(case["rot"], case["axes"], case["order"])
        st["freqs"], st["axis_of"] = f.cuda(), a.cuda()
        st["positions"] = _grid_positions(gen, case["axes"], B, L)
        return st
    dv = case["dv"]
    st["V"], st["log_decay"], st["scale"] = rows(Hk, dv), _log_decay(gen, case["decay"], Hk), d ** -0.5

    def states(n):          # those of texts of some tokens
        return torch.einsum("nhld,nhlv->nhdv", *(torch.randn((n, Hk, 12, w), generator=gen, device="cuda") for w in (d, dv)))

    if op == "train":
        st["dY"] = rows(H, dv)
        if case["initial"] == "own":
            st["before"], st["dafter"] = states(B), 0.1 * states(B)
        elif case["initial"] == "shared":
            st["before"], st["slots"] = states(1), torch.zeros((B,), dtype=torch.int32, device="cuda")
        return st
    # a pool with states to spare, the batch's in any order
    st["state"] = states(B + 3)
    st["slots"] = torch.randperm(B + 3, generator=gen, device="cuda")[:B].to(torch.int32)
    if op == "prompt":
        st["lengths"] = _lengths(gen, B, L)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def _own(st):
    from paper_2302_00787_amd import binding as fs
    case = st["case"]
    op = case["op"]
    if op == "turn":
        rot = fs.RotaryAxes(st["freqs"], st["axis_of"], st["positions"], case["interleaved"])
        return fs.rotary(st["Q"], rot, st["K"], transposed=case["transposed"])
    Q, K, V, g, scale = (st[x] for x in ("Q", "K", "V", "log_decay", "scale"))
    if op == "token":
        return fs.decay_step(st["state"], Q, K, V, g, scale, slots=st["slots"]), st["state"]
    if op == "prompt":
        pool = st["state"]
        return fs.decay_attention(Q, K, V, g, scale, before=None if case["fresh"] else pool, after=pool, lengths=st["lengths"],
                                  slots=st["slots"]), pool
    if case["initial"] == "none":
        return (fs.decay_attention(Q, K, V, g, scale),) + fs.decay_attention_backward(Q, K, V, st["dY"], g, scale)[:3]
    if case["initial"] == "shared":
        Y = fs.decay_attention(Q, K, V, g, scale, before=st["before"], slots=st["slots"])
        return (Y,) + fs.decay_attention_backward(Q, K, V, st["dY"], g, scale, before=st["before"], slots=st["slots"])
    after = torch.empty_like(st["before"])
    Y = fs.decay_attention(Q, K, V, g, scale, before=st["before"], after=after)
    return (Y, after) + fs.decay_attention_backward(Q, K, V, st["dY"], g, scale, before=st["before"], dafter=st["dafter"])


CHUNK = 128


def _powers(g, n):
    """lambda^n in 32 bits, the exponents in 64: g [Hk], n any whole numbers -> [Hk, *n.shape]."""
    return torch.exp(g.double().reshape(-1, *[1] * n.dim()) * n).float()


def _scan(g, x, a, b, first=None, before=None):
    """sum_(j <= i) lambda^(i-j) (x_i . a_j) b_j + lambda^(i + first) x_i before for x [B, Hk, G, L, .] and a, b [B, Hk, G, L, .] (either
    G may be one; the sum is over that of a and b too), in chunks: within them by their scores, between them by their states."""
    L, ones = x.shape[3], torch.arange(CHUNK, device="cuda")
    N = (L + CHUNK - 1) // CHUNK
    x, a, b = (torch.nn.functional.pad(t, (0, 0, 0, N * CHUNK - L)).unflatten(3, (N, CHUNK)) for t in (x, a, b))
    far = ones[:, None] - ones
    near = torch.where(far >= 0, _powers(g, far.clamp(min=0)), torch.zeros((), device="cuda"))
    y = (x @ a.transpose(-1, -2) * near[:, None, None]) @ b
    if a.shape[2] > 1:
        y = y.sum(2, keepdim=True)
    states = ((a * _powers(g, CHUNK - 1 - ones)[:, None, None, :, None]).transpose(-1, -2) @ b).sum(2)         # [B, Hk, N, ., .]
    n = torch.arange(N, device="cuda")
    gap = n[:, None] - 1 - n
    carry = torch.where(gap >= 0, _powers(g, CHUNK * gap.clamp(min=0)), torch.zeros((), device="cuda"))
    prefix = (carry @ states.flatten(3)).unflatten(3, states.shape[3:])
    inter = (x @ prefix[:, :, None]) * _powers(g, ones + 1)[:, None, None, :, None]
    y = (y + inter).flatten(3, 4)[:, :, :, :L]
    if before is not None:
        i = torch.arange(L, device="cuda")
        y = y + (x.flatten(3, 4)[:, :, :, :L] @ before[:, :, None]) * _powers(g, i + first)[:, None, :, None]
    return y


def _after(g, k, v, n, before):
    """The states after n [B] rows (k, v zero behind them) [B, Hk, L, .]."""
    j = torch.arange(k.shape[2], device="cuda")
    w = torch.exp(g.double()[None, :, None] * (n[:, None, None] - 1 - j).clamp(min=0)).float()
    S = (k * w[..., None]).transpose(-1, -2) @ v
    if before is not None:
        S = S + before * torch.exp(g.double() * n[:, None]).float()[..., None, None]
    return S


def run(st):
    if own:
        return _own(st)
    case = st["case"]
    op, dt = case["op"], _dtype(case)
    if op == "turn":
        return tuple(_turned(st, x).to(dt) for x in ("Q", "K"))
    B, Hk, L = case["B"], case["Hk"], case["L"]
    g, scale = st["log_decay"], st["scale"]
    q = st["Q"].float().unflatten(1, (Hk, -1))
    k, v = st["K"].float(), st["V"].float()
    if op == "train":
        return _train_plain(st, q, k, v)
    pool, at = st["state"], st["slots"].long()
    if op == "token":
        S = pool[at] * torch.exp(g)[:, None, None] + k.transpose(-1, -2) @ v
        pool[at] = S
        Y = (q @ S[:, :, None]) * scale
        return Y.flatten(1, 2).to(dt), pool
    behind = (torch.arange(L, device="cuda") >= st["lengths"][:, None])[:, None, :, None]
    k, v = k.masked_fill(behind, 0.0), v.masked_fill(behind, 0.0)
    before = None if case["fresh"] else pool[at]
    Y = _scan(g, q, k[:, :, None], v[:, :, None], 1, before) * scale
    pool[at] = _after(g, k, v, st["lengths"], before)
    return Y.flatten(1, 2).masked_fill(behind, 0.0).to(dt), pool


def _train_plain(st, q, k, v):
    case, dt, g, scale = st["case"], _dtype(st["case"]), st["log_decay"], st["scale"]
    B, Hk, L = case["B"], case["Hk"], case["L"]
    dy = st["dY"].float().unflatten(1, (Hk, -1))
    k1, v1 = k[:, :, None], v[:, :, None]
    before, after, dafter = st.get("before"), (), st.get("dafter")
    if "slots" in st:
        before = before[st["slots"].long()]
    Y = _scan(g, q, k1, v1, 1, before) * scale
    n = torch.full((B,), L, device="cuda")
    if case["initial"] == "own":
        after = (_after(g, k, v, n, before),)
    # queries: the same sums with dY, V, K in the places of Q, K, V; keys and values: from the last row to the first
    turned = None if before is None else before.transpose(-1, -2)
    dQ = _scan(g, dy, v1, k1, 1, turned) * scale
    qf, kf, vf, df = (t.flip(3) for t in (q * scale, k1, v1, dy))
    dK = _scan(g, vf, df, qf, 0, None if dafter is None else dafter.transpose(-1, -2)).flip(3)
    dV = _scan(g, kf, qf, df, 0, dafter).flip(3)
    out = (Y.flatten(1, 2).to(dt),) + after + (dQ.flatten(1, 2).to(dt), dK[:, :, 0].to(dt), dV[:, :, 0].to(dt))
    if before is None:
        return out
    i = torch.arange(L, device="cuda")
    dS = ((q * (_powers(g, i + 1) * scale)[:, None, :, None]).transpose(-1, -2) @ dy).sum(2)
    if dafter is not None:
        dS = dS + dafter * _powers(g, n[:1])[..., None]
    return out + (dS.sum(0, keepdim=True) if "slots" in st else dS,)


def _turned(st, name):
    """Rows in 32 bits turned by their positions, the angles in 64."""
    case, r, x = st["case"], st["case"]["rot"] // 2, st[name].float()
    places = st["positions"][st["axis_of"].long()].permute(1, 2, 0).double()          # [B, L, pairs]
    angle = (places * st["freqs"])[:, None]
    c, s = torch.cos(angle).float(), torch.sin(angle).float()
    if case["transposed"]:
        s = -s
    if case["interleaved"]:
        u, v = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
        turned = torch.stack([u * c - v * s, v * c + u * s], dim=-1).flatten(-2)
    else:
        u, v = x[..., :r], x[..., r:2 * r]
        turned = torch.cat([u * c - v * s, v * c + u * s], dim=-1)
    return torch.cat([turned, x[..., 2 * r:]], dim=-1)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    op = case["op"]
    if op != "turn" and case["B"] * case["H"] * case["L"] ** 2 * max(case["d"], case["dv"]) > 1 << 43:
        return None
    st = prepare(case, seed)
    if op == "turn":
        n = case["rot"]

        def turn(x):
            y = x.double()
            phase = torch.zeros((case["B"], case["L"], n // 2), dtype=torch.float64, device="cuda")
            for p, a in enumerate(st["axis_of"].tolist()):
                phase[:, :, p] = st["positions"][a] * st["freqs"][p]
            unit = torch.polar(torch.ones_like(phase), -phase if case["transposed"] else phase)[:, None]
            pairs = y[..., :n].unflatten(-1, (n // 2, 2)) if case["interleaved"] else y[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2)
            w = torch.view_as_real(torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * unit)
            y[..., :n] = (w if case["interleaved"] else w.transpose(-1, -2)).flatten(-2)
            return y

        return turn(st["Q"]), turn(st["K"])
    B, H, Hk, L, d, dv = (case[x] for x in ("B", "H", "Hk", "L", "d", "dv"))
    G, s = H // Hk, st["scale"]
    q, k, v, g = (st[x].double() for x in ("Q", "K", "V", "log_decay"))
    train = op == "train"
    pool = st["state"].double() if not train else None
    n = st["lengths"].tolist() if op == "prompt" else [L] * B
    Y = torch.zeros((B, H, L, dv), dtype=torch.float64, device="cuda")
    if train:
        dY = st["dY"].double()
        dQ, dK, dV = (torch.zeros_like(t) for t in (q, k, v))
        first = st["before"].double() if "before" in st else None
        last = torch.zeros((B, Hk, d, dv), dtype=torch.float64, device="cuda")
        dfirst = None if first is None else torch.zeros_like(first)
    for b in range(B):
        for h in range(Hk):
            m, lam, at = n[b], g[h], None
            if not train:
                at = int(st["slots"][b])
                S0 = torch.zeros_like(pool[at, h]) if case.get("fresh", False) else pool[at, h].clone()
            else:
                at = b if case["initial"] == "own" else 0
                S0 = None if first is None else first[at, h]
            t = torch.arange(m, dtype=torch.float64, device="cuda")
            for i0 in range(0, m, 2048):
                i1 = min(m, i0 + 2048)
                W = torch.exp(lam * (t[i0:i1, None] - t[None, :i1]).clamp(min=0.0)).tril(i0)
                grow = torch.exp(lam * (t[i0:i1, None] + 1.0))
                for e in range(h * G, (h + 1) * G):
                    A = s * W * (q[b, e, i0:i1] @ k[b, h, :i1].T)
                    Y[b, e, i0:i1] = A @ v[b, h, :i1]
                    if S0 is not None:
                        Y[b, e, i0:i1] += s * grow * (q[b, e, i0:i1] @ S0)
                    if train:
                        dA = s * W * (dY[b, e, i0:i1] @ v[b, h, :i1].T)
                        dQ[b, e, i0:i1] = dA @ k[b, h, :i1]
                        dK[b, h, :i1] += dA.T @ q[b, e, i0:i1]
                        dV[b, h, :i1] += A.T @ dY[b, e, i0:i1]
                        if S0 is not None:
                            dQ[b, e, i0:i1] += s * grow * (dY[b, e, i0:i1] @ S0.T)
                            dfirst[at, h] += s * (grow * q[b, e, i0:i1]).T @ dY[b, e, i0:i1]
            left = torch.exp(lam * (m - 1.0 - t))[:, None]
            S = (left * k[b, h, :m]).T @ v[b, h, :m]
            if S0 is not None:
                S += math.exp(lam * m) * S0
            if not train:
                pool[at, h] = S
            else:
                last[b, h] = S
                if "dafter" in st:
                    D = st["dafter"][b, h].double()
                    dK[b, h] += left * (v[b, h] @ D.T)
                    dV[b, h] += left * (k[b, h] @ D)
                    dfirst[at, h] += math.exp(lam * m) * D
    if not train:
        return Y, pool
    return (Y,) + ((last,) if case["initial"] == "own" else ()) + (dQ, dK, dV) + (() if first is None else (dfirst,))


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    """Inputs read once and outputs written once; multiply-adds of the recurrent form (two flops each), which no other form has fewer
    of: each key and each query meets a state once, in the backward pass the keys, the queries and their gradients do."""
    op, B, H, Hk, L, d = (case[x] for x in ("op", "B", "H", "Hk", "L", "d"))
    size = 2 if case["dtype"] == "bf16" else 4
    if op == "turn":
        rows = B * L * (H + Hk)
        return {"bytes": 2 * rows * d * size + 4 * case["axes"] * B * L, "flops": 3 * rows * case["rot"]}
    dv = case["dv"]
    state, rows, keys = 4 * Hk * d * dv, B * H * L, B * Hk * L
    if op == "token":
        return {"bytes": (rows + keys) * (d + dv) * size + 2 * B * state, "flops": 2 * (rows + keys) * d * dv}
    if op == "prompt":
        if B > 1:
            rows, keys = rows * 3 // 4, keys * 3 // 4     # a quarter of the batch is padding
        return {"bytes": (rows + keys) * (d + dv) * size + (1 if case["fresh"] else 2) * B * state, "flops": 2 * (rows + keys) * d * dv}
    kept = {"none": 0, "own": 4 * B, "shared": 2}[case["initial"]] * state
    return {"bytes": (rows * (2 * d + 2 * dv) + keys * 2 * (d + dv)) * size + kept, "flops": 2 * (3 * rows + 4 * keys) * d * dv}
