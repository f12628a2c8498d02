"""Pins of oracle/token_stats_oracle.py: closed forms, ties, central differences, and reverse-mode differentiation of an
independently written torch float64 form."""
import numpy as np
import pytest
import torch

from oracle.token_stats_oracle import token_stats, token_stats_backward


def _case(seed, T=6, d=9, V=23):
    g = np.random.default_rng(seed)
    y = g.integers(0, V, T)
    y[2] = -1
    return g.normal(0, 1.5, (T, d)), g.normal(0, 0.6, (V, d)), y, g.normal(0, 1, T), g.normal(0, 1, T)


def test_closed_forms():
    h, w = np.zeros((1, 4)), np.ones((10, 4))
    out = token_stats(h, w, [3], 0.7, 4)
    assert out["logprobs"][0] == pytest.approx(-np.log(10)) and out["entropy"][0] == pytest.approx(np.log(10))
    assert list(out["top_ids"][0]) == [0, 1, 2, 3]          # equal logits: the lower ids
    w = np.zeros((5, 4))
    w[3] = 100.0
    out = token_stats(np.ones((1, 4)), w, [3], 1.0, 2)
    assert out["logprobs"][0] == 0.0 and out["entropy"][0] == pytest.approx(0.0, abs=1e-12)
    assert list(out["top_ids"][0]) == [3, 0]


def test_against_torch_and_its_gradients():
    for seed in (0, 1, 2):
        h, w, y, gl, ge = _case(seed)
        out = token_stats(h, w, y, 0.7, 5)
        th, tw = (torch.tensor(x, requires_grad=True) for x in (h, w))
        logp = torch.log_softmax(th @ tw.T / 0.7, 1)
        ent = torch.distributions.Categorical(logits=th @ tw.T / 0.7).entropy()
        lp = torch.where(torch.tensor(y) >= 0, logp.gather(1, torch.tensor(y).clamp(min=0)[:, None])[:, 0], 0.0)
        np.testing.assert_allclose(out["logprobs"], lp.detach(), rtol=1e-12, atol=1e-12)
        np.testing.assert_allclose(out["entropy"], ent.detach(), rtol=1e-12)
        top = logp.topk(5, 1)
        assert (out["top_ids"] == top.indices.numpy()).all()
        np.testing.assert_allclose(out["top_logprobs"], top.values.detach(), rtol=1e-12)
        (torch.tensor(gl) * lp + torch.tensor(ge) * ent).sum().backward()
        dh, dw, _ = token_stats_backward(h, w, y, gl, ge, 0.7)
        np.testing.assert_allclose(dh, th.grad, rtol=1e-10, atol=1e-12)
        np.testing.assert_allclose(dw, tw.grad, rtol=1e-10, atol=1e-12)


def test_gradients_match_central_differences():
    h, w, y, gl, ge = _case(7)
    dh, dw, _ = token_stats_backward(h, w, y, gl, ge, 0.7)

    def loss():
        out = token_stats(h, w, y, 0.7)
        return float((gl * out["logprobs"] + ge * out["entropy"]).sum())

    g, eps = np.random.default_rng(3), 1e-6
    for arr, grad in ((h, dh), (w, dw)):
        for _ in range(12):
            i = tuple(g.integers(0, s) for s in arr.shape)
            old = arr[i]
            arr[i] = old + eps
            up = loss()
            arr[i] = old - eps
            down = loss()
            arr[i] = old
            assert grad[i] == pytest.approx((up - down) / (2 * eps), rel=1e-5, abs=1e-8)


def test_gradient_rows_sum_to_zero_over_the_vocabulary():
    h, w, y, gl, ge = _case(9)
    _, _, dl = token_stats_backward(h, w, y, gl, ge, 0.7)
    assert np.abs(dl.sum(1)).max() < 1e-12
