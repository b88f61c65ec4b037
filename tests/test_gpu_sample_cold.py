"""Sampling at temperatures of a few last places of the largest logit, where the border below which logits weigh nothing
falls between two neighbouring floats: every row gets the token and the probability of the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import serving as OS

pytestmark = pytest.mark.gpu

SENTINEL = -77


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _below(mx, ulps):
    x = np.float32(mx)
    for _ in range(ulps):
        x = np.nextafter(x, np.float32(-np.inf))
    return x


# logits in one crowded bin, a few, and a whole slice of them beyond the sorted candidates
@pytest.mark.parametrize("V,ties", [(64, 1), (3001, 700), (4096, 2500)])
@pytest.mark.parametrize("mx", [12.5, 8.0, 1.0, -3.7, 1000.0, 0.0])
@pytest.mark.parametrize("kw", [dict(top_p=0.9), dict(top_p=0.9999), dict(top_k=2), dict(top_k=2000, top_p=0.9999), dict(),
                                dict(min_p=1e-9)])
def test_temperatures_of_a_few_last_places(B, V, ties, mx, kw):
    rng = np.random.default_rng(V)
    temps = [1e-6, 3e-7, 1.2e-7, 5e-8, 1e-8, 1e-9, 1e-30]
    rows, temperature, us = [], [], []
    for t in temps:
        for ulps in (1, 2, 4, 8, 10, 12, 16):
            row = np.full(V, np.float32(mx) - np.float32(5), np.float32)
            at = rng.permutation(V)
            row[at[:ties]] = _below(mx, ulps)
            row[at[ties]] = mx
            rows.append(row)
            temperature.append(t)
            us.append(rng.random())
    pad = torch.zeros(len(rows), -(-V // 4) * 4, device="cuda")
    pad[:, :V] = torch.from_numpy(np.stack(rows)).cuda()
    M = len(rows)
    fill = lambda v, kind: torch.full((M,), v, dtype=kind, device="cuda")  # noqa: E731
    u = torch.tensor(us, device="cuda")
    tokens = fill(SENTINEL, torch.int32)
    args = dict(temperature=torch.tensor(temperature, device="cuda"),
                top_k=fill(kw["top_k"], torch.int32) if "top_k" in kw else None,
                **{n: fill(kw[n], torch.float32) if n in kw else None for n in ("top_p", "min_p")})
    got, prob = B.sample(pad[:, :V], u, tokens=tokens, want_probs=True, **args)
    got, prob = got.cpu().numpy(), prob.cpu().numpy()
    for r in range(M):
        t, p, _ = OS.sample(rows[r], float(u[r]), float(args["temperature"][r]), **kw)
        assert got[r] == t, (r, temperature[r], got[r], t)
        assert abs(prob[r] - p) <= 2.0 ** -22 * p + 1e-12  # one rounding to fp32, weights to 2^-27
