"""layer_norm and layer_norm_grads against the plain 64-bit form, with the bounds of
recognition_ref (counted roundings), and the gradient against central differences."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_1410_4984_amd as gpps  # noqa: E402
import recognition_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16}


def wide(kind):
    return torch.float64 if kind == "f64" else torch.float32


def f64(t):
    return t.detach().double().cpu().numpy()


def make(N, D, kind, seed=0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(N, D, generator=g, dtype=torch.float64) + shift).to(DT[kind]).to(DEV)
    dy = torch.randn(N, D, generator=g, dtype=torch.float64).to(DT[kind]).to(DEV)
    w = (1 + 0.3 * torch.randn(D, generator=g, dtype=torch.float64)).to(wide(kind)).to(DEV)
    b = torch.randn(D, generator=g, dtype=torch.float64).to(wide(kind)).to(DEV)
    return x, w, b, dy


def close(got, want, tol, what):
    d = np.abs(f64(got) - want)
    assert np.all(d <= tol), (what, float((d / np.maximum(tol, 1e-300)).max()))


# widths below one vector, one past a group's, odd ones, a row for each number of threads
WIDTHS = [1, 3, 8, 31, 33, 64, 129, 257, 333, 512, 1000, 1024, 2047, 4096, 6001, 16384]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f64"])
@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("N", [1, 37])
def test_forward_and_gradient(kind, D, N):
    x, w, b, dy = make(N, D, kind, seed=D + N)
    y, mean, rstd = gpps.layer_norm(x, w, b, 1e-5)
    assert y.dtype == x.dtype and mean.dtype == rstd.dtype == wide(kind)
    X, W, B = f64(x), f64(w), f64(b)
    ty, tm, tr = ref.layer_norm_tol(X, W, B, 1e-5, kind)
    ry, rm, rr = ref.layer_norm(X, W, B, 1e-5)
    close(y, ry, ty, "y")
    close(mean, rm, tm, "mean")
    close(rstd, rr, tr, "rstd")
    out = gpps.layer_norm_grads(x, w, mean, rstd, dy)
    want = ref.layer_norm_grads(X, W, f64(mean), f64(rstd), f64(dy))
    tol = ref.layer_norm_grads_tol(X, W, f64(mean), f64(rstd), f64(dy), kind)
    for k, r, t in zip(("dx", "dweight", "dbias"), want, tol):
        close(out[k], r, t, k)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f64"])
@pytest.mark.parametrize("D", [5, 48, 300, 1100])
def test_many_rows_sum_the_weights_gradient(kind, D):
    x, w, b, dy = make(3001, D, kind, seed=7)
    y, mean, rstd = gpps.layer_norm(x, w, b)
    out = gpps.layer_norm_grads(x, w, mean, rstd, dy)
    args = (f64(x), f64(w), f64(mean), f64(rstd), f64(dy))
    for k, r, t in zip(("dx", "dweight", "dbias"), ref.layer_norm_grads(*args),
                       ref.layer_norm_grads_tol(*args, kind)):
        close(out[k], r, t, k)
    # the same again, bit by bit
    again = gpps.layer_norm_grads(x, w, mean, rstd, dy)
    assert all(torch.equal(out[k], again[k]) for k in out)
    # added to, in two parts
    acc = gpps.layer_norm_grads(x[:1000], w, mean[:1000], rstd[:1000], dy[:1000])
    acc["dx"] = torch.empty_like(x[1000:])
    gpps.layer_norm_grads(x[1000:], w, mean[1000:], rstd[1000:], dy[1000:], accumulate=True, out=acc)
    tol = ref.layer_norm_grads_tol(*args, kind)
    for k, r, t in zip(("dweight", "dbias"), ref.layer_norm_grads(*args)[1:], tol[1:]):
        close(acc[k], r, t, k)


def test_large_mean_keeps_its_digits():
    """Rows of 1000 + noise: the variance is of the differences, so rstd keeps its digits."""
    x, w, b, dy = make(50, 700, "f32", seed=3, shift=1000.0)
    y, mean, rstd = gpps.layer_norm(x, w, b)
    ty, tm, tr = ref.layer_norm_tol(f64(x), f64(w), f64(b), 1e-5, "f32")
    ry, rm, rr = ref.layer_norm(f64(x), f64(w), f64(b), 1e-5)
    close(y, ry, ty, "y")
    # (x - mean is exact but for the mean's own rounding, which moves all differences alike)
    assert np.abs(f64(rstd) / rr - 1).max() < 1e-5


def test_without_weight_and_bias_and_strided():
    for kind in ("f32", "bf16", "f64"):
        x, w, b, dy = make(19, 77, kind, seed=5)
        wide_x = torch.zeros(19, 201, dtype=x.dtype, device=DEV)
        view = wide_x[:, 3:80]
        view.copy_(x)
        wide_y = torch.full((19, 99), 7.0, dtype=x.dtype, device=DEV)
        plain = gpps.layer_norm(x)
        stats = torch.empty(2, 19, dtype=wide(kind), device=DEV)
        gpps.layer_norm(view, out=(wide_y[:, 11:88], stats[0], stats[1]))
        assert torch.equal(wide_y[:, 11:88], plain[0]) and torch.equal(stats[0], plain[1])
        assert bool((wide_y[:, :11] == 7).all()) and bool((wide_y[:, 88:] == 7).all())
        ones, zeros = torch.ones_like(w), torch.zeros_like(b)
        assert torch.equal(plain[0], gpps.layer_norm(x, ones, zeros)[0])
        g1 = gpps.layer_norm_grads(x, ones, plain[1], plain[2], dy)
        g2 = gpps.layer_norm_grads(view, None, plain[1], plain[2], dy, bias=False)
        assert torch.equal(g1["dx"], g2["dx"]) and g2["dweight"] is None and g2["dbias"] is None
        # in place
        z = x.clone()
        gpps.layer_norm(z, w, b, out=(z, stats[0], stats[1]))
        assert torch.equal(z, gpps.layer_norm(x, w, b)[0])


def test_rows_do_not_mix():
    """A row with NaN or infinities, or of one value, leaves the others as they are."""
    x, w, b, dy = make(12, 40, "f32", seed=9)
    clean = gpps.layer_norm(x, w, b)[0]
    bad = x.clone()
    bad[3, 5], bad[4, 1], bad[5] = float("nan"), float("inf"), 2.0
    y, mean, rstd = gpps.layer_norm(bad, w, b)
    keep = [i for i in range(12) if i not in (3, 4, 5)]
    assert torch.equal(y[keep], clean[keep])
    assert bool(y[3].isnan().all()) and not bool(y[4].isfinite().any())
    assert torch.equal(y[5], b)                              # (x - mean) is zero, rstd finite


def test_no_rows():
    for kind in ("f32", "bf16", "f64"):
        x = torch.empty(0, 30, dtype=DT[kind], device=DEV)
        w = torch.ones(30, dtype=wide(kind), device=DEV)
        y, mean, rstd = gpps.layer_norm(x, w, w)
        assert y.shape == (0, 30) and mean.shape == (0,)
        out = gpps.layer_norm_grads(x, w, mean, rstd, x)
        assert bool((out["dweight"] == 0).all()) and bool((out["dbias"] == 0).all())
        out["dweight"].fill_(3)
        gpps.layer_norm_grads(x, w, mean, rstd, x, accumulate=True, out=out)
        assert bool((out["dweight"] == 3).all())


def test_gradient_against_differences():
    x, w, b, dy = make(5, 23, "f64", seed=11)
    y, mean, rstd = gpps.layer_norm(x, w, b)
    out = gpps.layer_norm_grads(x, w, mean, rstd, dy)

    def loss(x, w, b):
        return float((gpps.layer_norm(x, w, b)[0] * dy).sum())

    # central differences: e^2 of the third derivative (values of some tens here) and 2^-53 |L| / e
    e = 1e-5
    for t, k in ((x, "dx"), (w, "dweight"), (b, "dbias")):
        for i in range(0, t.numel(), 7):
            keep = float(t.view(-1)[i])
            t.view(-1)[i] = keep + e
            up = loss(x, w, b)
            t.view(-1)[i] = keep - e
            down = loss(x, w, b)
            t.view(-1)[i] = keep
            assert abs((up - down) / (2 * e) - float(out[k].view(-1)[i])) < 1e-7, (k, i)


def test_rows_past_32_bits():
    """The last rows of an array of more than 2^31 elements."""
    D, N = 2048, (1 << 20) + 40
    x = torch.zeros(N, D, dtype=torch.bfloat16, device=DEV)
    tail = make(40, D, "bf16", seed=13)
    x[-40:] = tail[0]
    y, mean, rstd = gpps.layer_norm(x, tail[1], tail[2])
    small = gpps.layer_norm(tail[0], tail[1], tail[2])
    assert torch.equal(y[-40:], small[0]) and torch.equal(rstd[-40:], small[2])
    dy = torch.zeros_like(x)
    dy[-40:] = tail[3]
    dx = gpps.layer_norm_grads(x, tail[1], mean, rstd, dy, out={"dx": y, "dweight": None, "dbias": None})["dx"]
    assert torch.equal(dx[-40:], gpps.layer_norm_grads(tail[0], tail[1], small[1], small[2], tail[3])["dx"])


def test_another_stream():
    x, w, b, dy = make(400, 512, "f32", seed=15)
    want = gpps.layer_norm(x, w, b)
    grads = gpps.layer_norm_grads(x, w, want[1], want[2], dy)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = gpps.layer_norm(x, w, b, stream=st)
    again = gpps.layer_norm_grads(x, w, got[1], got[2], dy, stream=st)
    st.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    assert all(torch.equal(again[k], grads[k]) for k in grads)


def test_refusals():
    x, w, b, dy = make(6, 16, "f32")
    with pytest.raises(ValueError):
        gpps.layer_norm(x.cpu())
    with pytest.raises(ValueError):
        gpps.layer_norm(x.t())                               # elements of a row are not neighbours
    with pytest.raises(ValueError):
        gpps.layer_norm(x[:1].expand(6, 16))                 # rows that overlap
    with pytest.raises(ValueError):
        gpps.layer_norm(x, w[:5])
    with pytest.raises(ValueError):
        gpps.layer_norm(x, w.double())
    with pytest.raises(TypeError):
        gpps.layer_norm(x.half())
    with pytest.raises(gpps.GppsError) as e:
        gpps.layer_norm(x, w, b, float("nan"))
    assert e.value.status == 3
    with pytest.raises(gpps.GppsError) as e:
        gpps.layer_norm(torch.zeros(2, 16385, device=DEV))
    assert e.value.status == 2
    y, mean, rstd = gpps.layer_norm(x, w, b)
    with pytest.raises(ValueError):
        gpps.layer_norm_grads(x, w, mean[:3], rstd, dy)
    with pytest.raises(ValueError):
        gpps.layer_norm_grads(x, w, mean, rstd, dy, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))


def test_sums_over_millions_of_rows():
    """float32 sums over so many rows that there are more workgroups than usual."""
    N, D = 7_000_003, 300
    x = torch.randn(N, D, device=DEV)
    y, mean, rstd = gpps.layer_norm(x)
    dy = y.fill_(0.1)
    out = gpps.layer_norm_grads(x, torch.ones(D, device=DEV), mean, rstd, dy)
    tenth = float(torch.tensor(0.1))
    exact, size = torch.zeros(D, dtype=torch.float64, device=DEV), torch.zeros(D, dtype=torch.float64, device=DEV)
    for part in torch.arange(N, device=DEV).split(1_000_000):
        t = tenth * (x[part].double() - mean[part, None].double()) * rstd[part, None].double()
        exact += t.sum(0)
        size += t.abs().sum(0)
    # a thread adds some 2,048 terms one by one at most, the rest in 64 slices and trees: fewer than 3,000 roundings
    # on the longest way
    tol = 3000 * 2.0 ** -24
    assert float((out["dbias"].double() - N * tenth).abs().max()) < tol * N * tenth
    assert bool(((out["dweight"].double() - exact).abs() < tol * size).all())
