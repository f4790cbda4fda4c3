"""The operators of a recognition model's training, as they are measured.

A recognition model gives q(x_n) of the GP-LVM as a function of the data: rows of
sequences pass a layer norm and a gated linear recurrence, the bound's gradients
come back through both, and AdamW updates every tensor of the model.

  ln_fwd   layer norm over the rows of x [N, D]: y, mean, rstd
  ln_bwd   its gradients: dx, dweight, dbias
  rec_fwd  h_t = a_t h_{t-1} + (1 - a_t) x_t, a = sigmoid(gate), over packed sequences
           (rows offsets[b] .. offsets[b+1]-1 are sequence b): h, h_last
  rec_bwd  its gradients: dx, dgate, dh0
  adamw    one step over many tensors, the two moments held in 32 (64) or in 8 bits

``own`` selects the framework's kernels; otherwise the plain form runs, elementary
torch operations in 32 bits (64 for float64 inputs), rounded once at the end.
Row counts are those of the framework's workloads (one row, a minibatch of
sequences, the 50,000 to 131,072 rows of its data sets); widths are a recognition
network's.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
DT = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f64": 8, "bf16": 2}
BLOCK = 256          # elements of a tensor that share one scale of an 8-bit state
EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


def listed():
    return [
        # serving: the norm of one new row, where the call's latency is all
        {"name": "ln_fwd_one", "kind": "ln_fwd", "dtype": "f32", "N": 1, "D": 512},
        # an ordinary data set through a wide layer in mixed precision
        {"name": "ln_fwd_bf16", "kind": "ln_fwd", "dtype": "bf16", "N": 50000, "D": 1024},
        # training in the fits' default type, an odd width
        {"name": "ln_bwd_f64", "kind": "ln_bwd", "dtype": "f64", "N": 5001, "D": 333},
        # a row chunk of the million-row workload through the widest layer
        {"name": "ln_bwd_bf16", "kind": "ln_bwd", "dtype": "bf16", "N": 131072, "D": 2048},
        # streaming: one new row for each of 64 sequences, with carried states
        {"name": "rec_fwd_step", "kind": "rec_fwd", "dtype": "f32", "N": 64, "D": 512, "seqs": 64,
         "lengths": "one", "reverse": False, "carry": True},
        # the headline data set as 500 sequences of ragged lengths, empty ones among them
        {"name": "rec_fwd_ragged", "kind": "rec_fwd", "dtype": "f32", "N": 100000, "D": 256, "seqs": 500,
         "lengths": "ragged", "reverse": False, "carry": True},
        # one unbroken recording of 131,072 rows, mixed precision
        {"name": "rec_fwd_long", "kind": "rec_fwd", "dtype": "bf16", "N": 131072, "D": 1024, "seqs": 1,
         "lengths": "ragged", "reverse": False, "carry": False},
        # the smoothing direction's gradient: few long sequences, an odd width
        {"name": "rec_bwd_odd", "kind": "rec_bwd", "dtype": "bf16", "N": 50001, "D": 301, "seqs": 37,
         "lengths": "ragged", "reverse": True, "carry": True},
        # the largest training batch in single precision
        {"name": "rec_bwd_f32", "kind": "rec_bwd", "dtype": "f32", "N": 131072, "D": 1024, "seqs": 64,
         "lengths": "ragged", "reverse": False, "carry": False},
        # a small recognition network: a dozen tensors, launches and host time
        {"name": "adamw_small", "kind": "adamw", "dtype": "f32", "grad": "f32", "bits": 32, "tensors": 14,
         "total": 400000},
        # a large one, states in 32 bits, gradients from mixed precision
        {"name": "adamw_32", "kind": "adamw", "dtype": "f32", "grad": "bf16", "bits": 32, "tensors": 150,
         "total": 100000000},
        # the same with its states in 8 bits
        {"name": "adamw_8", "kind": "adamw", "dtype": "f32", "grad": "f32", "bits": 8, "tensors": 150,
         "total": 100000000},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: N 1 .. 131,072, D 8 .. 4,096, sequences of one row to all rows; 1 to 200
    tensors of 1,000 to 100 million elements together."""
    kind = rng.choice(["ln_fwd", "ln_bwd", "rec_fwd", "rec_bwd", "adamw"])
    if kind == "adamw":
        dtype, grad = rng.choice([("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"),
                                  ("f64", "f64")])
        bits = 64 if dtype == "f64" else rng.choice([8, 32])
        total = _log_int(rng, 1000, 50000000 if dtype == "f64" else 100000000)
        return {"kind": kind, "dtype": dtype, "grad": grad, "bits": bits,
                "tensors": _log_int(rng, 1, max(1, min(200, total // 100))), "total": total}
    case = {"kind": kind, "dtype": rng.choice(["f32", "bf16", "f64"]), "D": _log_int(rng, 8, 4096)}
    most = 131072 * 1024 * 4 // SIZE[case["dtype"]]          # elements of one array
    case["N"] = _log_int(rng, 1, min(131072, most // case["D"]))
    if kind in ("rec_fwd", "rec_bwd"):
        case["lengths"] = rng.choice(["ragged", "ragged", "ragged", "one"])
        case["seqs"] = case["N"] if case["lengths"] == "one" else _log_int(rng, 1, case["N"])
        case["reverse"] = rng.random() < 0.5
        case["carry"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ inputs

def _tensor_sizes(case):
    """Element counts of the tensors: matrices of uneven size and, every other one, a vector."""
    n, total = case["tensors"], case["total"]
    r = random.Random(n * 1000003 + total)
    weight = [r.uniform(0.001, 0.01) if i % 2 else r.uniform(0.5, 4.0) for i in range(n)]
    sizes = [max(1, int(total * w / sum(weight))) for w in weight]
    sizes[0] += max(0, total - sum(sizes))
    return sizes


def _wide(dt):
    """The type of sums, states and parameters beside arrays of type dt."""
    return torch.float64 if dt == torch.float64 else torch.float32


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind, dt = case["kind"], DT[case["dtype"]]

    def randn(*shape, dtype=None):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dtype or dt)

    s = {"kind": kind}
    if kind == "adamw":
        # each tensor begins at a multiple of 256 elements, as the allocator places it; what lies
        # between two tensors stays zero
        sizes = _tensor_sizes(case)
        starts, at = [], 0
        for n in sizes:
            starts.append(at)
            at += -(-n // BLOCK) * BLOCK
        inside = torch.zeros(at, dtype=torch.bool, device=DEV)
        for a, n in zip(starts, sizes):
            inside[a:a + n] = True
        wide = _wide(dt)
        flat = {"p": (0.02 * randn(at)) * inside, "g": (1e-3 * randn(at, dtype=DT[case["grad"]])) * inside}
        m = 3e-4 * randn(at, dtype=wide) * inside
        v = 1e-6 * randn(at, dtype=wide).square() * inside
        if case["bits"] == 8:
            # codes spread as a running fit leaves them, and the scales of its blocks
            unit = torch.rand(at, generator=g, device=DEV)
            sign = torch.where(m < 0, -1.0, 1.0)
            flat["m"] = (sign * (127 * unit).round() * inside).to(torch.int8)
            flat["v"] = ((40 + 215 * torch.rand(at, generator=g, device=DEV)).round() * inside).to(torch.uint8)
            blocks = at // BLOCK
            flat["m_scale"] = 1e-3 * (0.5 + torch.rand(blocks, generator=g, device=DEV))
            flat["v_scale"] = 1e-5 * (0.5 + torch.rand(blocks, generator=g, device=DEV))
        else:
            flat["m"], flat["v"] = m, v
        s["flat"] = flat
        s["tensors"] = {k: [f[a // BLOCK:-(-(a + n) // BLOCK)] if k.endswith("scale") else f[a:a + n]
                            for a, n in zip(starts, sizes)] for k, f in flat.items()}
        s["step"] = 100
        return s
    N, D, wide = case["N"], case["D"], _wide(dt)
    if kind in ("ln_fwd", "ln_bwd"):
        # activations with an offset and a spread of their own in each row
        x = randn(N, D, dtype=torch.float32)
        s["x"] = (x * (0.5 + torch.rand(N, 1, generator=g, device=DEV)) + 0.5 * randn(N, 1, dtype=torch.float32)).to(dt)
        s["weight"] = 1 + 0.1 * randn(D, dtype=wide)
        s["bias"] = 0.1 * randn(D, dtype=wide)
        if kind == "ln_bwd":
            xw = s["x"].to(wide)
            s["mean"] = xw.mean(1)
            s["rstd"] = 1 / ((xw - s["mean"][:, None]).square().mean(1) + EPS).sqrt()
            s["dy"] = randn(N, D)
        return s
    B = case["seqs"]
    if case["lengths"] == "one":
        cuts = torch.arange(B + 1, device=DEV)
    else:
        inner = torch.randint(0, N + 1, (B - 1,), generator=g, device=DEV).sort().values
        ends = torch.tensor([0, N], device=DEV)
        cuts = torch.cat([ends[:1], inner, ends[1:]])
    s["offsets"], s["reverse"] = cuts, case["reverse"]
    s["x"] = randn(N, D)
    # memories of about two to some hundred rows
    s["gate"] = (2.5 + 1.5 * randn(N, D, dtype=torch.float32)).to(dt)
    s["h0"] = randn(B, D, dtype=wide) if case["carry"] else None
    if kind == "rec_bwd":
        s["h"] = _plain_rec_fwd(s)[0]
        s["dh"] = randn(N, D)
        s["dh_last"] = randn(B, D, dtype=wide) if case["carry"] else None
    return s


# ------------------------------------------------------------------ plain forms

def _plain_ln_fwd(s):
    x = s["x"].to(s["weight"].dtype)
    mean = x.sum(1) / x.shape[1]
    xc = x - mean[:, None]
    rstd = 1 / torch.sqrt((xc * xc).sum(1) / x.shape[1] + EPS)
    y = xc * rstd[:, None] * s["weight"] + s["bias"]
    return [y.to(s["x"].dtype), mean, rstd]


def _plain_ln_bwd(s):
    wide = s["weight"].dtype
    D = s["x"].shape[1]
    dy = s["dy"].to(wide)
    xh = (s["x"].to(wide) - s["mean"][:, None]) * s["rstd"][:, None]
    u = dy * s["weight"]
    dx = s["rstd"][:, None] * (u - u.sum(1, keepdim=True) / D - xh * ((u * xh).sum(1, keepdim=True) / D))
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xh).sum(0), "dbias": dy.sum(0)}


def _rows(s):
    """Per row: its sequence, and whether it is the first or the last one taken; per sequence: whether it has rows."""
    off, N = s["offsets"], s["x"].shape[0]
    row = torch.arange(N, device=off.device)
    seq = torch.searchsorted(off[1:].contiguous(), row, right=True)
    low, high = row == off[seq], row == off[seq + 1] - 1
    first, last = (high, low) if s["reverse"] else (low, high)
    return seq, first[:, None], last[:, None], (off[1:] > off[:-1])[:, None]


def _last_rows(s):
    off = s["offsets"]
    return (off[:-1] if s["reverse"] else off[1:] - 1).clamp(0, s["x"].shape[0] - 1)


def _linear_scan(a, b):
    """y_t = a_t y_{t-1} + b_t over dim 0, by doubling the number of rows that each row covers."""
    k, N = 1, a.shape[0]
    while k < N:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _plain_rec_fwd(s):
    wide = _wide(s["x"].dtype)
    x, gate = s["x"].to(wide), s["gate"].to(wide)
    seq, first, last, some = _rows(s)
    a, b = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
    u = b * x
    if s["h0"] is not None:
        u = torch.where(first, u + a * s["h0"][seq], u)
    a = torch.where(first, 0, a)
    h = _linear_scan(a.flip(0), u.flip(0)).flip(0) if s["reverse"] else _linear_scan(a, u)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros_like(h[:1])
    h_last = torch.where(some, h[_last_rows(s)], h0)
    return [h.to(s["x"].dtype), h_last]


def _plain_rec_bwd(s):
    wide = _wide(s["x"].dtype)
    x, gate, h, dh = (s[k].to(wide) for k in ("x", "gate", "h", "dh"))
    seq, first, last, some = _rows(s)
    a, b = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
    off = s["offsets"]
    zero = torch.zeros_like(h[:1])
    if s["dh_last"] is not None:
        dh = torch.where(last, dh + s["dh_last"][seq], dh)
    # G_t = dh_t + a_next G_next, from the last row taken to the first
    if s["reverse"]:
        before = torch.cat([h[1:], zero])
        G = _linear_scan(torch.where(last, 0, torch.cat([zero, a[:-1]])), dh)
    else:
        before = torch.cat([zero, h[:-1]])
        G = _linear_scan(torch.where(last, 0, torch.cat([a[1:], zero])).flip(0), dh.flip(0)).flip(0)
    before = torch.where(first, s["h0"][seq] if s["h0"] is not None else 0, before)
    at = (off[1:] - 1 if s["reverse"] else off[:-1]).clamp(0, x.shape[0] - 1)
    dh0 = torch.where(some, a[at] * G[at], s["dh_last"] if s["dh_last"] is not None else 0)
    return {"dx": (b * G).to(s["x"].dtype), "dgate": (a * b * G * (before - x)).to(s["x"].dtype), "dh0": dh0}


def _values(m, v, m_scale, v_scale):
    """What 8-bit states stand for, as rows of one block each."""
    c = m.reshape(-1, BLOCK).to(torch.float32)
    r = c.abs() * (1.0 / 127.0)
    q = v.reshape(-1, BLOCK).to(torch.float32) * (1.0 / 255.0)
    q2 = q * q
    return m_scale[:, None] * (r * r) * torch.sign(c), v_scale[:, None] * (q2 * q2)


def _codes(m, v):
    """8-bit states and their scales of moments in rows of one block each."""
    tiny = torch.finfo(torch.float32).tiny
    sm, sv = m.abs().amax(1, keepdim=True), v.amax(1, keepdim=True)
    sm, sv = torch.where(sm < tiny, 0, sm), torch.where(sv < tiny, 0, sv)
    im, iv = torch.where(sm == 0, 0, 1 / sm), torch.where(sv == 0, 0, 1 / sv)
    cm = torch.round(torch.sqrt(m.abs() * im) * 127) * torch.sign(m)
    cv = torch.round(torch.sqrt(torch.sqrt(v * iv)) * 255)
    cv = torch.where((v > 0) & (sv > 0), cv.clamp(min=1), cv)
    return cm.to(torch.int8), cv.to(torch.uint8), sm[:, 0], sv[:, 0]


def _plain_adamw(s):
    f, wide = s["flat"], _wide(s["flat"]["p"].dtype)
    eight = "m_scale" in f
    s["step"] += 1
    p, g = f["p"].to(wide), f["g"].to(wide)
    m, v = _values(f["m"], f["v"], f["m_scale"], f["v_scale"]) if eight else (f["m"], f["v"])
    m = m.reshape(-1) * BETA1 + g * (1 - BETA1)
    v = v.reshape(-1) * BETA2 + g * (1 - BETA2) * g
    denom = torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** s["step"])) + ADAM_EPS
    p = p * (1 - LR * DECAY) - m / denom * (LR / (1 - BETA1 ** s["step"]))
    f["p"].copy_(p)
    if not eight:
        f["m"].copy_(m)
        f["v"].copy_(v)
        return {"p": f["p"], "m": f["m"], "v": f["v"]}
    cm, cv, sm, sv = _codes(m.reshape(-1, BLOCK), v.reshape(-1, BLOCK))
    f["m"].copy_(cm.reshape(-1))
    f["v"].copy_(cv.reshape(-1))
    f["m_scale"].copy_(sm)
    f["v_scale"].copy_(sv)
    m, v = _values(cm, cv, sm, sv)
    return {"p": f["p"], "m": m.reshape(-1), "v": v.reshape(-1)}


PLAIN = {"ln_fwd": _plain_ln_fwd, "ln_bwd": _plain_ln_bwd, "rec_fwd": _plain_rec_fwd,
         "rec_bwd": _plain_rec_bwd, "adamw": _plain_adamw}


# ------------------------------------------------------------------ the framework's calls

def run(s):
    if not own:
        return PLAIN[s["kind"]](s)
    import paper_1410_4984_amd as gpps
    kind = s["kind"]
    if kind == "ln_fwd":
        return list(gpps.layer_norm(s["x"], s["weight"], s["bias"], EPS))
    if kind == "ln_bwd":
        return gpps.layer_norm_grads(s["x"], s["weight"], s["mean"], s["rstd"], s["dy"])
    if kind == "rec_fwd":
        return list(gpps.recurrence(s["x"], s["gate"], s["offsets"], s["h0"], reverse=s["reverse"]))
    if kind == "rec_bwd":
        return gpps.recurrence_grads(s["x"], s["gate"], s["h"], s["dh"], s["offsets"], s["h0"], s["dh_last"],
                                     reverse=s["reverse"])
    t, f = s["tensors"], s["flat"]
    s["step"] += 1
    gpps.adamw_step(t["p"], t["g"], t["m"], t["v"], s["step"], LR, betas=(BETA1, BETA2), eps=ADAM_EPS,
                    weight_decay=DECAY, m_scale=t.get("m_scale"), v_scale=t.get("v_scale"))
    if "m_scale" not in f:
        return {"p": f["p"], "m": f["m"], "v": f["v"]}
    return {"p": f["p"], "m": gpps.adamw_values(f["m"], f["m_scale"]), "v": gpps.adamw_values(f["v"], f["v_scale"])}


# ------------------------------------------------------------------ work

def work(case):
    kind, e = case["kind"], SIZE[case["dtype"]]
    w = 8 if case["dtype"] == "f64" else 4                    # statistics, states, parameters
    if kind == "adamw":
        n, eg = case["total"], SIZE[case["grad"]]
        if case["bits"] == 8:
            # codes in and out, a scale per block and moment in and out, and the values returned
            return {"bytes": n * (2 * e + eg + 4 + 8) + 16 * (n // BLOCK), "flops": 30 * n}
        return {"bytes": n * (2 * e + eg + 4 * w), "flops": 14 * n}
    N, D = case["N"], case["D"]
    if kind == "ln_fwd":
        return {"bytes": 2 * N * D * e + 2 * N * w + 2 * D * w, "flops": 8 * N * D}
    if kind == "ln_bwd":
        return {"bytes": 3 * N * D * e + 2 * N * w + 3 * D * w, "flops": 14 * N * D}
    B = case["seqs"]
    states = B * D * w * (2 if case["carry"] else 1) + 8 * (B + 1)
    if kind == "rec_fwd":
        return {"bytes": 3 * N * D * e + states, "flops": 8 * N * D}
    return {"bytes": 6 * N * D * e + states + (B * D * w if case["carry"] else 0), "flops": 14 * N * D}


# ------------------------------------------------------------------ 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    f64, kind = torch.float64, case["kind"]

    if kind in ("ln_fwd", "ln_bwd"):
        x = s["x"].to(f64)
        D = x.shape[1]
        if kind == "ln_fwd":
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = (var + EPS) ** -0.5
            return [torch.addcmul(s["bias"].to(f64), (x - mean[:, None]) * rstd[:, None], s["weight"].to(f64)), mean, rstd]
        # with mean and rstd as given; the row's Jacobian applied to u = dy * weight
        xh = (x - s["mean"].to(f64)[:, None]) * s["rstd"].to(f64)[:, None]
        dy = s["dy"].to(f64)
        u = dy * s["weight"].to(f64)
        along = torch.linalg.vecdot(u, xh, dim=1)[:, None] / D
        dx = (u - u.mean(1, keepdim=True) - along * xh) * s["rstd"].to(f64)[:, None]
        return {"dx": dx, "dweight": torch.linalg.vecdot(dy, xh, dim=0), "dbias": dy.sum(0)}

    if kind in ("rec_fwd", "rec_bwd"):
        N, D = s["x"].shape
        x, gate = s["x"].to(f64), s["gate"].to(f64)
        off = s["offsets"].tolist()
        B = len(off) - 1
        back = s["reverse"]
        live = [b for b in range(B) if off[b + 1] > off[b]]
        begin = torch.tensor([off[b + 1] - 1 if back else off[b] for b in live], device=DEV)
        end = torch.tensor([off[b] if back else off[b + 1] - 1 for b in live], device=DEV)
        which = torch.tensor(live, device=DEV)
        a = torch.sigmoid(gate)
        h0 = s["h0"].to(f64) if s["h0"] is not None else torch.zeros(B, D, dtype=f64, device=DEV)

        def steps(a, u):
            # y_t = a_t y_{t-1} + u_t in rows: blocks of about sqrt(N) rows side by side, step by
            # step, then the blocks' ends one after the other, then both joined
            C = max(1, math.isqrt(N))
            K = -(-N // C)
            pad = K * C - N
            a = torch.cat([a, a.new_zeros(pad, D)]).view(K, C, D)
            y = torch.cat([u, u.new_zeros(pad, D)]).view(K, C, D).clone()
            A = a.clone()
            for t in range(1, C):
                y[:, t] += a[:, t] * y[:, t - 1]
                A[:, t] *= A[:, t - 1]
            for k in range(1, K):
                y[k] += A[k] * y[k - 1, -1]
            return y.view(K * C, D)[:N]

        if kind == "rec_fwd":
            u = torch.sigmoid(-gate) * x
            u[begin] += a[begin] * h0[which]
            a[begin] = 0
            h = steps(a.flip(0), u.flip(0)).flip(0) if back else steps(a, u)
            h_last = h0.clone()
            h_last[which] = h[end]
            return [h, h_last]
        h = s["h"].to(f64)
        before = torch.zeros_like(h)
        if back:
            before[:-1] = h[1:]
        else:
            before[1:] = h[:-1]
        before[begin] = h0[which]
        dl = s["dh_last"].to(f64) if s["dh_last"] is not None else torch.zeros_like(h0)
        u = s["dh"].to(f64)
        u[end] += dl[which]
        nxt = torch.zeros_like(a)                             # a of the row taken after this one
        if back:
            nxt[1:] = a[:-1]
        else:
            nxt[:-1] = a[1:]
        nxt[end] = 0
        G = steps(nxt, u) if back else steps(nxt.flip(0), u.flip(0)).flip(0)
        dh0 = dl.clone()
        dh0[which] = a[begin] * G[begin]
        return {"dx": torch.sigmoid(-gate) * G, "dgate": G * (before - x) * a * torch.sigmoid(-gate), "dh0": dh0}

    f = s["flat"]
    t = s["step"] + 1
    p, g = f["p"].to(f64), f["g"].to(f64)
    if case["bits"] == 8:
        c = f["m"].to(f64)
        m = f["m_scale"].to(f64).repeat_interleave(BLOCK) * c * c.abs() / 127 ** 2
        v = f["v_scale"].to(f64).repeat_interleave(BLOCK) * (f["v"].to(f64) / 255) ** 4
    else:
        m, v = f["m"].to(f64), f["v"].to(f64)
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g ** 2, v, BETA2)
    p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + ADAM_EPS)
    if case["bits"] == 8:
        sm = m.abs().view(-1, BLOCK).amax(1).repeat_interleave(BLOCK)
        sv = v.view(-1, BLOCK).amax(1).repeat_interleave(BLOCK)
        cm = (127 * (m.abs() / sm) ** 0.5).nan_to_num(0).round()
        cv = (255 * (v / sv) ** 0.25).nan_to_num(0).round()
        cv = torch.where(v > 0, cv.clamp(min=1), cv)
        m, v = torch.sign(m) * sm * (cm / 127) ** 2, sv * (cv / 255) ** 4
    return {"p": p, "m": m, "v": v}
