"""The recognition model (paper_1410_4984_amd.recognition): every operator together, as a fit runs them.

CPU: the bounds of sequences that come from the host.  GPU: the network's gradients
against differences of the bound, a fit on sequences of a one-dimensional latent, and
streaming against whole sequences."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_1410_4984_amd as gpps  # noqa: E402
from paper_1410_4984_amd import recognition  # noqa: E402

DEV = "cuda:0"


def sequences(lengths, seed=0, noise=0.05):
    """Rows of sequences whose latent swings along one curve in three dimensions (the same curve for
    every seed), an RBF draw as in section 4.  Returns (Y, x, offsets)."""
    rng = np.random.default_rng(seed)
    x = np.concatenate([2.5 * np.sin(rng.uniform(0.02, 0.08) * np.arange(n) + rng.uniform(0, 2 * np.pi))
                        for n in lengths])
    g = np.linspace(-3.5, 3.5, 512)
    K = np.exp(-0.5 * (g[:, None] - g[None]) ** 2)
    F = np.linalg.cholesky(K + 1e-10 * np.eye(512)) @ np.random.default_rng(7).normal(size=(512, 3))
    Y = np.stack([np.interp(x, g, F[:, d]) for d in range(3)], 1)
    return Y + noise * rng.normal(size=Y.shape), x, np.concatenate([[0], np.cumsum(lengths)])


def test_offsets_from_the_host_are_checked():
    cpu = torch.device("cpu")
    assert recognition._offsets(None, 5, cpu) is None
    assert recognition._offsets([0, 0, 3, 5], 5, cpu).tolist() == [0, 0, 3, 5]
    for bad in ([0, 4], [1, 5], [0, 3, 2, 5], [5], [[0, 5]]):
        with pytest.raises(ValueError):
            recognition._offsets(bad, 5, cpu)


def rank_correlation(a, b):
    rank = lambda v: np.argsort(np.argsort(v))  # noqa: E731
    return np.corrcoef(rank(a), rank(b))[0, 1]


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_against_differences_of_the_bound(causal):
    Y, _, offsets = sequences([0, 25, 1, 14], seed=1)
    N, Q, M = Y.shape[0], 2, 6
    model = recognition.Recognizer(3, Q, 7, causal=causal, dtype=torch.float64, seed=3,
                                   projection=np.random.default_rng(4).normal(size=(3, Q)))
    Yt = torch.tensor(Y, device=DEV)
    off = torch.tensor(offsets, device=DEV)
    Z = torch.tensor(np.random.default_rng(5).normal(size=(M, Q)), device=DEV)

    def evaluate():
        mu, logS, kept, _ = model.forward(Yt, off)
        S = logS.exp()
        return gpps.bound(mu, S, Z, Yt, 1.2, [1.0, 0.8], 5.0, 1e-4), S, kept

    out, S, kept = evaluate()
    grads = model.backward(kept, out["dmu"], out["dS"] * S)
    rng = np.random.default_rng(6)
    # central differences: e^2 of the third derivative, and the bound's own rounding over e
    e = 1e-5
    for name, w in model.weights.items():
        flat = w.view(-1)
        for i in rng.choice(flat.numel(), size=min(6, flat.numel()), replace=False):
            keep = float(flat[i])
            flat[i] = keep + e
            up = float(evaluate()[0]["L"])
            flat[i] = keep - e
            down = float(evaluate()[0]["L"])
            flat[i] = keep
            got = float(grads[name].reshape(-1)[i])
            assert abs((up - down) / (2 * e) - got) <= 1e-5 * (1 + abs(got)), (name, i)


@pytest.mark.gpu
@pytest.mark.parametrize("causal,bits", [(False, 32), (True, 8)])
def test_fit_recovers_the_latent_of_new_sequences(causal, bits):
    Y, x, offsets = sequences([0, 300, 1, 500, 700, 0, 499])
    r = recognition.fit(Y, 1, 20, offsets=offsets, steps=300, bits=bits, causal=causal, hidden=48)
    mu, S = r.model.infer(Y, offsets)
    new, x_new, new_offsets = sequences([400, 350], seed=5)
    mu_new, S_new = r.model.infer(new, new_offsets)
    rho = rank_correlation(mu[:, 0].cpu().numpy(), x)
    rho_new = rank_correlation(mu_new[:, 0].cpu().numpy(), x_new)
    print(f"  L {r.bound_trace[0]:.0f} -> {r.bound_trace[-1]:.0f}, rank correlation {rho:.3f}, of new "
          f"sequences {rho_new:.3f}, beta {r.beta:.1f}, {1e3 * r.seconds / len(r.bound_trace):.2f} ms a step", flush=True)
    assert len(r.bound_trace) == 300 and r.bound_trace[-1] > r.bound_trace[0] + 1000.0
    assert abs(rho) > 0.9 and abs(rho_new) > 0.85
    assert bool((S > 0).all()) and bool((S_new > 0).all()) and bool(mu_new.isfinite().all())


@pytest.mark.gpu
def test_streaming_is_the_whole_sequence_row_by_row():
    model = recognition.Recognizer(3, 2, 16, causal=True, dtype=torch.float64, seed=2)
    lengths = [60] * 4
    Y, _, offsets = sequences(lengths, seed=8)
    mu, S = model.infer(Y, offsets)
    rows = torch.tensor(Y).view(4, 60, 3)
    state = None
    for t in range(60):
        m, s, state = model.stream(rows[:, t], state)
        # sums of a few dozen terms in another order
        assert float((m - mu.view(4, 60, 2)[:, t]).abs().max()) < 1e-12
        assert float((s - S.view(4, 60, 2)[:, t]).abs().max()) < 1e-12
    with pytest.raises(ValueError):
        recognition.Recognizer(3, 2, 16).stream(rows[:, 0])
