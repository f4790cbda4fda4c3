"""adamw_step and AdamW against the plain 64-bit step, with the bounds of
recognition_ref, and the 8-bit moments against the same codes computed in numpy,
every operation rounded once in 32 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_1410_4984_amd as gpps  # noqa: E402
import recognition_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16}
HYPER = (1e-2, 0.9, 0.99, 1e-8, 0.02)      # lr, betas, eps, weight decay

# one element, one more than a vector and a block, none, several workgroups; over 64 tensors
SIZES = [1, 5, 255, 256, 257, 0, 2048, 2049, 10001, 64] + [3] * 60 + [777]
TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f64", "f64")]


def f64(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def tensors(kind, grad, seed=0, sizes=SIZES):
    g = torch.Generator().manual_seed(seed)
    w = torch.float64 if kind == "f64" else torch.float32

    def make(dtype, scale, fn=lambda t: t):
        return [fn(scale * torch.randn(n, generator=g, dtype=torch.float64)).to(dtype).to(DEV) for n in sizes]

    return make(DT[kind], 0.1), make(DT[grad], 1e-2), make(w, 1e-2), make(w, 1e-2, lambda t: t.square())


@pytest.mark.parametrize("kind,grad", TYPES)
@pytest.mark.parametrize("maximize", [False, True])
def test_against_the_plain_step(kind, grad, maximize):
    p, g, m, v = tensors(kind, grad)
    lr, b1, b2, eps, wd = HYPER
    for step in (1, 2, 1000):
        args = [[f64(t) for t in ts] for ts in (p, g, m, v)]
        gpps.adamw_step(p, g, m, v, step, lr, betas=(b1, b2), eps=eps, weight_decay=wd, maximize=maximize)
        for i in range(len(p)):
            a = [args[0][i], -args[1][i] if maximize else args[1][i], args[2][i], args[3][i]]
            want = ref.adamw(*a, step, lr, b1, b2, eps, wd)
            tol = ref.adamw_tol(*a, step, lr, b1, b2, eps, wd, kind)
            for t, r, e, name in zip((p, m, v), want, tol, "pmv"):
                d = np.abs(f64(t[i]) - r)
                assert np.all(d <= e), (step, i, name, float((d / np.maximum(e, 1e-300)).max()))


def blocks(t):
    """A tensor's values as rows of one block, filled with zeros."""
    t = t.detach().cpu().numpy().reshape(-1)
    return np.concatenate([t, np.zeros(-t.size % 256, t.dtype)]).reshape(-1, 256)


def test_codes_of_8_bits_are_exact():
    for kind, grad in (("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")):
        p, g, _, _ = tensors(kind, grad, seed=2)
        opt = gpps.AdamW(p, 1e-2, betas=(0.9, 0.99), bits=8)
        b1, c1, b2, c2 = (np.float32(c) for c in (0.9, 1 - 0.9, 0.99, 1 - 0.99))
        for step in range(4):
            before = [(blocks(a), blocks(b), s.cpu().numpy(), t.cpu().numpy())
                      for a, b, s, t in zip(opt.m, opt.v, opt.m_scale, opt.v_scale)]
            old = [f64(t) for t in p]
            opt.step(g)
            for i in range(len(p)):
                if not p[i].numel():
                    continue
                cm, cv, sm, sv = before[i]
                gr = blocks(g[i].float())
                m32, v32 = ref.values_m(cm, sm), ref.values_v(cv, sv)
                m = m32 * b1 + gr * c1
                v = v32 * b2 + gr * c2 * gr
                n = p[i].numel()
                want = ref.encode(m, v)
                assert np.array_equal(blocks(opt.m[i]), want[0]) and np.array_equal(blocks(opt.v[i]), want[1])
                assert np.array_equal(opt.m_scale[i].cpu().numpy(), want[2])
                assert np.array_equal(opt.v_scale[i].cpu().numpy(), want[3])
                # what the codes stand for
                assert np.array_equal(blocks(gpps.adamw_values(opt.m[i], opt.m_scale[i])), ref.values_m(*want[::2]))
                assert np.array_equal(blocks(gpps.adamw_values(opt.v[i], opt.v_scale[i])), ref.values_v(*want[1::2]))
                # the step uses the moments before they are rounded
                a = (old[i], f64(g[i]), *(t.reshape(-1)[:n].astype(np.float64) for t in (m32, v32)))
                want_p = ref.adamw(*a, step + 1, 1e-2, 0.9, 0.99, 1e-8, 0.01)[0]
                tol = ref.adamw_tol(*a, step + 1, 1e-2, 0.9, 0.99, 1e-8, 0.01, kind)[0]
                assert np.all(np.abs(f64(p[i]) - want_p) <= tol), (step, i)
            g = [t.roll(1) * 0.7 for t in g]


def test_codes_at_the_ends():
    """Blocks of zeros, of one value, of tiny values, one large value among small ones; a v above
    zero never gets the code of zero."""
    n = 256 * 5
    g = torch.zeros(n, device=DEV)
    g[256:512] = 1e-3
    g[512:768] = 1e-25                                       # its square is below the normal range
    g[768:1024] = 1e-6
    g[800] = 1.0
    g[1024:] = -torch.linspace(0, 1, 256, device=DEV)
    p = torch.ones(n, device=DEV)
    opt = gpps.AdamW([p], 1e-3, bits=8)
    opt.step([g])
    m, v = opt.m[0].view(5, 256), opt.v[0].view(5, 256)
    assert bool((m[0] == 0).all()) and bool((v[0] == 0).all()) and float(opt.m_scale[0][0]) == 0
    assert bool((m[1] == 127).all()) and bool((v[1] == 255).all())
    assert bool((v[2] == 0).all()) and float(opt.v_scale[0][2]) == 0
    assert int(v[3, 32]) == 255 and bool((v[3] >= 1).all())
    assert bool((m[4] <= 0).all()) and int(m[4, -1]) == -127
    assert bool(p.isfinite().all())
    for _ in range(3):
        opt.step([g])
    assert bool(p.isfinite().all())


def test_a_block_that_is_not_finite():
    """NaN or infinite gradients show in their block's moments and nowhere else."""
    g = torch.full((1024,), 1e-2, device=DEV)
    clean = gpps.AdamW([torch.ones(1024, device=DEV)], 1e-3, bits=8)
    opt = gpps.AdamW([torch.ones(1024, device=DEV)], 1e-3, bits=8)
    bad = g.clone()
    bad[300], bad[700] = float("nan"), float("inf")
    opt.step([bad])
    opt.step([g])
    clean.step([g])
    clean.step([g])
    for o, codes, scale in ((opt.m[0], opt.m, opt.m_scale), (opt.v[0], opt.v, opt.v_scale)):
        val = gpps.adamw_values(codes[0], scale[0]).view(4, 256)
        assert bool(val[1].isnan().all()) and not bool(val[2].isfinite().any())
    keep = [0, 3]
    assert torch.equal(opt.params[0].view(4, 256)[keep], clean.params[0].view(4, 256)[keep])
    assert torch.equal(opt.m[0].view(4, 256)[keep], clean.m[0].view(4, 256)[keep])


@pytest.mark.parametrize("bits", [32, 8])
def test_odd_addresses_and_neighbours(bits):
    """Tensors that begin at odd elements of a larger one; what lies around them stays."""
    for dtype in (torch.float32, torch.bfloat16):
        n, pad = 3001, 7
        big = {k: torch.full((n + 2 * pad,), 9, dtype=t, device=DEV) for k, t in
               (("p", dtype), ("g", dtype), ("m", torch.int8 if bits == 8 else torch.float32),
                ("v", torch.uint8 if bits == 8 else torch.float32))}
        part = {k: t[pad:pad + n] for k, t in big.items()}
        part["p"].copy_(torch.randn(n, device=DEV))
        part["g"].copy_(1e-2 * torch.randn(n, device=DEV))
        part["m"].zero_()
        part["v"].zero_()
        scales = [torch.zeros(-(-n // 256), device=DEV) for _ in range(2)] if bits == 8 else [None, None]
        own = {k: t.clone() for k, t in part.items()}
        more = [t.clone() if t is not None else None for t in scales]

        def step(d, s):
            gpps.adamw_step([d["p"]], [d["g"]], [d["m"]], [d["v"]], 1, 1e-2, m_scale=None if s[0] is None else [s[0]],
                            v_scale=None if s[1] is None else [s[1]])

        step(part, scales)
        step(own, more)
        assert all(torch.equal(part[k], own[k]) for k in part)
        assert all(bool((t[:pad] == 9).all()) and bool((t[pad + n:] == 9).all()) for t in big.values())


def test_mixed_types_missing_gradients_and_lr():
    """One list with several types; a tensor without a gradient is left; lr of one step."""
    p = [torch.ones(10, dtype=t, device=DEV) for t in (torch.float32, torch.float64, torch.bfloat16, torch.float32)]
    g = [torch.full_like(t, 0.5) for t in p]
    g[3] = None
    opt = gpps.AdamW(p, 1e-3, weight_decay=0.0)
    opt.step(g, lr=0.125)
    # the first step is lr g / |g|
    assert abs(float(p[0][0]) - 0.875) < 1e-6 and abs(float(p[1][0]) - 0.875) < 1e-7
    assert abs(float(p[2][0]) - 0.875) <= 2.0 ** -9 and float(p[3][0]) == 1.0
    assert opt.steps == 1 and bool((opt.m[3] == 0).all())
    up = gpps.AdamW([torch.ones(3, device=DEV)], 0.125, weight_decay=0.0, maximize=True)
    up.step([torch.full((3,), 0.5, device=DEV)])
    assert abs(float(up.params[0][0]) - 1.125) < 1e-6


def test_past_32_bits():
    """The end of a tensor of more than 2^31 elements."""
    n = (1 << 31) + 1000
    p = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    tail = 256 * 3 + (n % 256)
    p[-tail:] = torch.randn(tail, device=DEV).to(torch.bfloat16)
    g[-tail:] = torch.randn(tail, device=DEV).to(torch.bfloat16)
    small = gpps.AdamW([p[-tail:].clone()], 1e-2, bits=8)
    small.step([g[-tail:].clone()])
    big = gpps.AdamW([p], 1e-2, bits=8)
    big.step([g])
    assert torch.equal(p[-tail:], small.params[0])
    assert torch.equal(big.m[0][-tail:], small.m[0]) and torch.equal(big.v[0][-tail:], small.v[0])
    assert bool((p[:1000] == 0).all())


def test_another_stream():
    p, g, m, v = tensors("f32", "f32", seed=4)
    q, n, w = ([t.clone() for t in ts] for ts in (p, m, v))
    gpps.adamw_step(p, g, m, v, 3, 1e-2)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    gpps.adamw_step(q, g, n, w, 3, 1e-2, stream=st)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(p + m + v, q + n + w))


def test_8_bits_follow_32():
    """A least-squares fit reaches the same loss with either kind of moments."""
    g = torch.Generator().manual_seed(5)
    X = torch.randn(400, 50, generator=g).to(DEV)
    y = X @ torch.randn(50, 1, generator=g).to(DEV)
    loss = {}
    for bits in (32, 8):
        w = torch.zeros(50, 1, device=DEV)
        opt = gpps.AdamW([w], 0.05, weight_decay=0.0, bits=bits)
        for _ in range(300):
            opt.step([X.t() @ (X @ w - y) / 400])
        loss[bits] = float((X @ w - y).square().mean())
    start = float(y.square().mean())
    assert loss[32] < 1e-3 * start and loss[8] < 1e-3 * start, loss


def test_refusals():
    p, g, m, v = tensors("f32", "f32", sizes=[8, 9])
    with pytest.raises(ValueError):
        gpps.adamw_step(p, g[:1], m, v, 1, 1e-3)
    with pytest.raises(ValueError):
        gpps.adamw_step([t.cpu() for t in p], g, m, v, 1, 1e-3)
    with pytest.raises(ValueError):
        gpps.adamw_step(p, [t.cpu() for t in g], m, v, 1, 1e-3)
    with pytest.raises(ValueError):
        gpps.adamw_step(p, g, [t[:4] for t in m], v, 1, 1e-3)
    with pytest.raises(ValueError):
        gpps.adamw_step(p, g, [t.bfloat16() for t in m], v, 1, 1e-3)
    with pytest.raises(ValueError):
        gpps.adamw_step([p[0], p[0]], [g[0], g[0]], [m[0], m[0]], [v[0], v[0]], 1, 1e-3)
    with pytest.raises(ValueError):
        gpps.adamw_step([torch.zeros(4, 6, device=DEV).t()], [torch.zeros(6, 4, device=DEV)],
                        [torch.zeros(6, 4, device=DEV)], [torch.zeros(6, 4, device=DEV)], 1, 1e-3)
    with pytest.raises(TypeError):
        gpps.adamw_step(p, [t.double() for t in g], m, v, 1, 1e-3)
    with pytest.raises(TypeError):
        gpps.AdamW([torch.zeros(4, dtype=torch.float64, device=DEV)], bits=8).step(
            [torch.zeros(4, dtype=torch.float64, device=DEV)])
    for bad in ({"lr": float("nan")}, {"lr": -1.0}, {"lr": 1e-3, "betas": (1.0, 0.9)}, {"lr": 1e-3, "eps": -1.0},
                {"lr": 1e-3, "weight_decay": float("inf")}):
        with pytest.raises(gpps.GppsError) as e:
            gpps.adamw_step(p, g, m, v, 1, **bad)
        assert e.value.status == 3
    with pytest.raises(gpps.GppsError) as e:
        gpps.adamw_step(p, g, m, v, 0, 1e-3)
    assert e.value.status == 2
    keep = [t.clone() for t in p]
    assert all(torch.equal(a, b) for a, b in zip(p, keep))
