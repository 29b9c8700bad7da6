"""Oracle pins of the scored step and of the orthogonalised update: finite differences, torch's own log_softmax, singular values."""
import numpy as np
import pytest

from hift_inputs import WORKLOADS, init_params, make_batch, model_config
from oracle import hift_oracle as O


def test_scores_against_torch_and_differences():
    import torch
    g = np.random.default_rng(0)
    x, y = g.standard_normal((7, 31)) * 2, np.array([0, 30, -1, 5, 31, 7, 7])
    logp, ent = O.token_scores(x, y, 0.8)
    ref = torch.distributions.Categorical(logits=torch.from_numpy(0.8 * x))
    has = (y >= 0) & (y < 31)
    assert np.allclose(ent, ref.entropy().numpy(), atol=1e-13) and (logp[~has] == 0).all()
    assert np.allclose(logp[has], ref.log_prob(torch.from_numpy(np.where(has, y, 0))).numpy()[has], atol=1e-13)
    dl, dh = g.standard_normal(7), g.standard_normal(7)
    d = O.token_scores_bwd(x, y, 0.8, dl, dh)
    for j in range(31):
        e = np.zeros_like(x)
        e[:, j] = 1e-5
        (a, b), (c, f) = O.token_scores(x + e, y, 0.8), O.token_scores(x - e, y, 0.8)
        assert np.allclose((dl * (a - c) + dh * (b - f)) / 2e-5, d[:, j], atol=1e-8)


def test_loss_is_a_score():
    wl = WORKLOADS["C1"]
    cfg = model_config(wl)
    theta = init_params(1, [(n, s, k) for n, s, k, _u in O.param_tensors(cfg)], bf16_exact=False).astype(np.float64)
    tok, lab = make_batch(wl, 1, 1)
    loss, g = O.loss_and_grad(cfg, theta, tok, lab)
    n = (lab >= 0).sum()

    def objective(logits, rows):
        return -O.token_scores(logits, rows)[0].sum() / n, O.token_scores_bwd(logits, rows, 1.0, np.full(rows.size, -1.0 / n), np.zeros(rows.size))

    loss2, g2 = O.loss_and_grad(cfg, theta, tok, lab, objective=objective)
    assert abs(loss - loss2) < 1e-12 and np.allclose(g, g2, atol=1e-14)


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (6, 6), (1, 7), (7, 1)])
def test_orthogonalize_maps_singular_values(shape):
    u = np.random.default_rng(2).standard_normal(shape) * 1e-3
    q, s, v = np.linalg.svd(u, full_matrices=False)
    s = s / np.linalg.norm(u)
    a, b, c = O.MUON_COEFFICIENTS
    for _ in range(O.MUON_STEPS):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(O.orthogonalize(u), (q * s) @ v, atol=1e-12) and s.max() < 1.3 and s.min() > 0.6
    assert (O.orthogonalize(np.zeros(shape)) == 0).all()


def test_muon_update_by_hand_and_its_parts():
    theta, buf, g = np.full((1, 4), 2.0), np.full((1, 4), 1.0), np.full((1, 4), 0.5)
    O.muon_update(theta, g, buf, lr=0.1, momentum=0.9, wd=0.5)
    x = 0.5                                   # 1 x 4, all alike: its one singular value starts at 1
    a, b, c = O.MUON_COEFFICIENTS
    s = 1.0
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(buf, 1.4) and np.allclose(theta, 2.0 * 0.95 - 0.1 * 0.2 * 2.0 * x * s)
    cfg = model_config(WORKLOADS["C4"])
    parts = {n: O.muon_parts(n, s, u, cfg) for n, s, _k, u in O.param_tensors(cfg)}
    assert parts["l0.wqkv"] == [(0, 4096), (4096, 8192), (8192, 12288)] and parts["l3.wgu"] == [(0, 11008), (11008, 22016)]
    assert parts["l0.wd"] == [(0, 4096)] and parts["l0.wo"] == [(0, 4096)] and not parts["l0.g1"] and not parts["tok_emb"] and not parts["whead"]
