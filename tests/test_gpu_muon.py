"""Orthogonalised updates on the GPU against float64, through the binding.

Bar of an orthogonalisation of five steps, 2-norm: each step rounds X, A and B to fp16 for its products, by 2^-11 / sqrt(3) of their values
(rms) at most, 2.8e-4.  Near the singular values the iteration settles at, X carries that into a step with the factor |B| <= 2.8, A with |b
+ 2 c A| s^2 <= 3 and B with 1; in quadrature 4.2 x 2.8e-4 = 1.2e-3 a step.  Steps pass earlier errors on by |a + 3 b s^2 + 5 c s^4| <= 1.2
there, and five add up, in quadrature, to at most 2.7e-3 x 1.2 = 3.3e-3.  Rounding to bfloat16 adds 2^-8 / sqrt(3) = 2.3e-3 at most: 4e-3
together.  Where the shorter side is below 16 the few singular values do not average their errors, which add in full: 1.5e-2."""
import numpy as np
import pytest

import paper_2403_17031_amd as P
from oracle.muon_oracle import muon_step, newton_schulz

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.load_library()
    return P


def _bar(shape):
    return 4e-3 if min(shape) >= 16 else 1.5e-2


def _matrix(rows, cols, kind, seed):
    g = np.random.default_rng(seed)
    if kind == "gauss":
        return 1e-4 * g.normal(0, 1, (rows, cols))
    if kind == "low":  # few strong directions over a floor of weak ones
        r = min(rows, cols) // 16 + 1
        return 1e-4 * (g.normal(0, 1, (rows, r)) @ g.normal(0, 1, (r, cols)) + 0.05 * g.normal(0, 1, (rows, cols)))
    if kind == "steep":  # rows and columns of very different sizes
        return g.normal(0, 1, (rows, cols)) * np.exp(-6 * np.arange(cols) / cols) * np.exp(-6 * np.arange(rows) / rows)[:, None]
    return g.normal(0, 1, (rows, 1)) @ g.normal(0, 1, (1, cols)) * 1e3  # one direction


def _off(have, want):
    return float(np.linalg.norm(have - want) / np.linalg.norm(want))


SHAPES = [(1, 1), (1, 300), (300, 1), (5, 7), (16, 16), (64, 64), (65, 63), (63, 65), (77, 1000), (1000, 77), (130, 130), (128, 512), (512, 128),
          (333, 1025), (1025, 333), (700, 2048)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind", ["gauss", "low", "steep", "one"])
def test_against_the_oracle(rows, cols, kind):
    import torch
    x = torch.from_numpy(_matrix(rows, cols, kind, rows + cols)).to("cuda", torch.float32)
    got = P.orthogonalize(x)
    assert got.dtype == torch.bfloat16 and got.shape == x.shape
    assert _off(got.double().cpu().numpy(), newton_schulz(x.double().cpu().numpy())) <= _bar((rows, cols))


@pytest.mark.parametrize("steps", [1, 2, 3, 10])
def test_other_numbers_of_steps(steps):
    import torch
    x = torch.from_numpy(_matrix(100, 260, "gauss", 1)).to("cuda", torch.float32)
    # (the bar's last line: one step's error in quadrature with those before, of which no more than five matter)
    assert _off(P.orthogonalize(x, ns_steps=steps).double().cpu().numpy(), newton_schulz(x.double().cpu().numpy(), steps)) <= 5e-3


def test_a_batch_is_its_matrices():
    """Also more of them than go together, and bfloat16 and in place."""
    import torch
    x = torch.stack([torch.from_numpy(_matrix(70, 130, "low", i)) for i in range(51)]).to("cuda", torch.bfloat16)
    one = torch.stack([P.orthogonalize(m) for m in x])
    assert (P.orthogonalize(x) == one).all()
    assert _off(one[50].double().cpu().numpy(), newton_schulz(x[50].double().cpu().numpy())) <= 4e-3
    y = x.clone()
    assert P.orthogonalize(y, out=y) is y and (y == one).all()
    assert P.orthogonalize(x[:0]).shape == (0, 70, 130)


def test_more_elements_than_go_together():
    """Nine matrices of 33.6 M elements, seven of which fill the workspace: the eighth and ninth share its second filling."""
    import torch
    n = 5800
    x = 1e-3 * torch.randn(9, n, n, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    got = P.orthogonalize(x)
    for i in (0, 6, 7, 8):
        assert torch.equal(got[i], P.orthogonalize(x[i]))
    X = x[8].double() / (x[8].double().norm() + 1e-7)
    for _ in range(5):
        A = X @ X.T.contiguous()
        X = 3.4445 * X + (-4.7750 * A + 2.0315 * (A @ A)) @ X
    assert float((got[8].double() - X).norm() / X.norm()) <= 4e-3


def test_nothing_infinities_and_tiny_values():
    import torch
    x = torch.zeros(4, 70, 90, device="cuda")
    x[1] = torch.from_numpy(_matrix(70, 90, "gauss", 5)).to("cuda", torch.float32)
    x[2] = x[1]
    x[2, 3, 4] = float("nan")
    x[3] = x[1] * 1e20  # norms beyond what fp32 squares hold
    got = P.orthogonalize(x)
    assert (got[0] == 0).all() and got[2].isnan().any()
    assert _off(got[1].double().cpu().numpy(), newton_schulz(x[1].double().cpu().numpy())) <= 4e-3
    assert _off(got[3].double().cpu().numpy(), newton_schulz(x[3].double().cpu().numpy())) <= 4e-3
    small = x[1] * 1e-25
    got = P.orthogonalize(small, eps=1e-30)
    assert _off(got.double().cpu().numpy(), newton_schulz(small.double().cpu().numpy(), eps=1e-30)) <= 4e-3


def _tensors(shapes, seed):
    import torch
    g = np.random.default_rng(seed)
    p = [torch.from_numpy(g.normal(0, 0.02, s)).to("cuda", torch.float32) for s in shapes]
    grad = [torch.from_numpy(_matrix(*s, "low", seed + i)).to("cuda", torch.float32) for i, s in enumerate(shapes)]
    m = [torch.from_numpy(0.3 * _matrix(*s, "low", seed + 50 + i)).to("cuda", torch.float32) for i, s in enumerate(shapes)]
    return p, grad, m, [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes]


def _np(ts):
    return [t.double().cpu().numpy() for t in ts]


@pytest.mark.parametrize("nesterov", [True, False])
def test_step_against_the_oracle(nesterov):
    """More tensors than go together, of all orientations, one of them empty; the parameters' move is compared, 2-norm."""
    import torch
    shapes = [(64, 64), (128, 40), (40, 128), (0, 5), (1, 33), (33, 1), (192, 64), (65, 200)] * 7
    p, grad, m, b = _tensors(shapes, 3)
    p0, g0, m0 = _np(p), _np(grad), _np(m)
    kw = dict(lr=0.05, momentum=0.9, nesterov=nesterov, weight_decay=0.1, rms=0.3, grad_scale=0.5)
    P.muon_step(p, grad, m, params_bf16=b, **kw)
    for i, s in enumerate(shapes):
        if 0 in s:
            continue
        want_p, want_m, _ = muon_step(p0[i], g0[i], m0[i], **kw)
        have = p[i].double().cpu().numpy()
        decayed = p0[i] * (1 - 0.05 * 0.1)
        assert _off(have - decayed, want_p - decayed) <= _bar(s), s
        # two products and their sum, half an ulp each
        assert (np.abs(m[i].double().cpu().numpy() - want_m) <= 2.0**-22 * (np.abs(m0[i]) + np.abs(g0[i]))).all()
        assert torch.equal(b[i], p[i].to(torch.bfloat16)) and (grad[i].double().cpu().numpy() == g0[i]).all()


def test_step_of_unaligned_views_and_without_copies():
    """Parameters at any float of a flat buffer, as the same step of separate arrays."""
    import torch
    shapes = [(65, 63), (32, 96), (7, 5)]
    p, grad, m, _ = _tensors(shapes, 9)
    flat = [torch.zeros(3 + sum(t.numel() + 1 for t in p), device="cuda") for _ in range(3)]
    views = []
    for f, ts in zip(flat, (p, grad, m)):
        at, vs = 3, []
        for t in ts:
            v = f[at:at + t.numel()].view(t.shape)
            v.copy_(t)
            vs.append(v)
            at += t.numel() + 1
        views.append(vs)
    P.muon_step(p, grad, m, lr=0.1)
    P.muon_step(*views, lr=0.1)
    for a, b in zip(p + m, views[0] + views[2]):
        assert torch.equal(a, b)
    for f, ts in zip(flat, (p, grad, m)):  # what lies between the views is as it was
        assert (f[:3] == 0).all()
        at = 3
        for t in ts:
            at += t.numel()
            assert f[at] == 0
            at += 1


def test_a_matrix_that_is_not_numbers_stays_alone():
    import torch
    shapes = [(64, 96)] * 3
    p, grad, m, b = _tensors(shapes, 4)
    q, h, n, c = _tensors(shapes, 4)
    h[1][5, 6] = float("inf")
    P.muon_step(p, grad, m, lr=0.1, params_bf16=b)
    P.muon_step(q, h, n, lr=0.1, params_bf16=c)
    for i in (0, 2):
        assert torch.equal(p[i], q[i]) and torch.equal(m[i], n[i]) and torch.equal(b[i], c[i])
    assert not torch.isfinite(q[1]).all()


def test_steps_repeat_themselves_on_poisoned_memory(monkeypatch):
    import torch
    monkeypatch.setattr(P.binding, "POISON", True)
    runs = []
    for _ in range(2):
        p, grad, m, b = _tensors([(100, 70), (70, 300)], 6)
        for _ in range(3):
            P.muon_step(p, grad, m, lr=0.1, params_bf16=b)
        runs.append(p + m + b + [P.orthogonalize(grad[0])])
    assert all(torch.equal(x, y) and torch.isfinite(x).all() for x, y in zip(*runs))


def test_another_stream_and_a_captured_graph():
    import torch
    shapes = [(64, 200), (200, 64), (130, 130)]
    p, grad, m, b = _tensors(shapes, 7)
    q, h, n, c = _tensors(shapes, 7)
    r, k, o, d = _tensors(shapes, 7)
    P.muon_step(p, grad, m, lr=0.1, params_bf16=b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.muon_step(q, h, n, lr=0.1, params_bf16=c)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(p + m + b, q + n + c))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        P.muon_step(r, k, o, lr=0.1, params_bf16=d)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        if i:
            P.muon_step(p, grad, m, lr=0.1, params_bf16=b)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(p + m + b, r + o + d)), i


def test_refusals_of_the_binding():
    import torch
    a = torch.zeros(4, 6, device="cuda")
    for bad in (lambda: P.orthogonalize(a.half()), lambda: P.orthogonalize(a.T), lambda: P.orthogonalize(a[0]), lambda: P.orthogonalize(a, ns_steps=0),
                lambda: P.orthogonalize(a, out=a), lambda: P.orthogonalize(a, eps=0.0),
                lambda: P.muon_step([a], [a.clone()], [a[:2].clone()]), lambda: P.muon_step([a], [a.clone()], [a.clone()], momentum=1.0),
                lambda: P.muon_step([a.T], [a.T], [a.T]), lambda: P.muon_step([a, a], [a.clone()] * 2, [a.clone(), a.clone()]),
                lambda: P.muon_step([a], [a.clone()], [a.clone()], params_bf16=[a]), lambda: P.muon_step([a.bfloat16()], [a], [a])):
        with pytest.raises(P.RlhfError):
            bad()
    P.muon_step([], [], [])
