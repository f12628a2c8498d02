"""Token statistics and their gradient on the GPU against float64, through the binding.

Inputs lie on a grid that every type holds and on which every sum of products is exact in fp32 (|h| < 8 in sixteenths, |w| < 1/8 in
1024ths: 24 bits hold a sum of 4096 such products), so that logits have one value, ids are comparable, and what is left is the
softmax's arithmetic.  Its bars: z = l / T is rounded twice, half an ulp each, 2^-23 |z|; exp is off by 2^-22 (1 + |x|) of its
value, weighted by values that fall as exp x, so by less than 2^-21 of the sum; a part's 64 terms and the V / 64 parts are added in fp32,
2^-24 of the sum each.  An entropy sums terms of up to |log p| + H times as much, but the same errors enter its two sums."""
import numpy as np
import pytest

import paper_2403_17031_amd as P
from oracle.token_stats_oracle import token_stats as oracle_stats
from oracle.token_stats_oracle import token_stats_backward as oracle_backward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.load_library()
    return P


def _dt(name):
    import torch
    return dict(fp32=torch.float32, bf16=torch.bfloat16, fp16=torch.float16)[name]


def _inputs(T, d, V, dtype, seed, lean=1.0):
    """float64 numpy (hidden, weight, targets) on the grid, and the CUDA tensors of them."""
    import torch
    g = np.random.default_rng(seed)
    w = np.clip(np.round(g.normal(0, 0.04, (V, d)) * 1024), -127, 127) / 1024
    y = g.integers(0, V, T)
    h = g.normal(0, 1, (T, d)) + lean * 12.0 * g.random((T, 1)) * w[y] / (0.0016 * d)
    h = np.clip(np.round(h * 16), -127, 127) / 16
    y = np.where(g.random(T) < 0.2, -1, y).astype(np.int32)
    dev = [torch.from_numpy(a).to("cuda", _dt(dtype)) for a in (h, w)]
    return h, w, y, dev[0], dev[1], torch.from_numpy(y).cuda()


def _check(got, h, w, y, temp, k):
    V = w.shape[0]
    want = oracle_stats(h, w, y, temp, k)
    zmax = np.abs(h @ w.T).max(1) / temp
    tol = 2.0**-22 * zmax + 2.0**-21 + (100 + V / 64) * 2.0**-24
    lp, ent, lse = (got[n].cpu().numpy().astype(np.float64) for n in ("logprobs", "entropy", "lse"))
    assert (np.abs(lse - want["lse"]) <= tol).all(), np.abs(lse - want["lse"]).max()
    assert (np.abs(lp - want["logprobs"]) <= 2 * tol).all()
    assert (lp[y < 0] == 0).all()
    assert (np.abs(ent - want["entropy"]) <= 2 * tol * (1 + want["entropy"])).all(), np.abs(ent - want["entropy"]).max()
    assert ("top_ids" in got) == (k > 0)
    if k:
        assert (got["top_ids"].cpu().numpy() == want["top_ids"]).all()
        assert (np.abs(got["top_logprobs"].cpu().numpy() - want["top_logprobs"]) <= 2 * tol[:, None]).all()


SIZES = [  # T, d, V, type, alternatives
    (1, 64, 100, "bf16", 3), (1, 1, 1, "fp32", 1), (2, 5, 3, "fp16", 3), (3, 37, 77, "fp16", 5), (5, 64, 64, "fp32", 64),
    (7, 32, 65, "fp32", 2), (17, 128, 1000, "bf16", 20), (31, 2560, 300, "bf16", 4), (33, 72, 129, "bf16", 64),
    (64, 768, 4099, "fp16", 0), (65, 96, 515, "fp32", 1), (130, 96, 130, "fp16", 0), (300, 520, 3001, "fp16", 12), (1030, 64, 2049, "bf16", 7),
    (4200, 64, 777, "fp16", 2), (17000, 64, 200, "bf16", 3), (66000, 64, 70, "fp16", 0),
]


@pytest.mark.parametrize("T,d,V,dtype,k", SIZES)
def test_against_the_oracle(T, d, V, dtype, k):
    h, w, y, th, tw, ty = _inputs(T, d, V, dtype, T + d + V)
    _check(P.token_stats(th, tw, ty, 0.7, k), h, w, y, 0.7, k)


@pytest.mark.parametrize("T,dtype", [(1, "bf16"), (19, "fp16"), (257, "bf16"), (1100, "fp16"), (40, "fp32")])
def test_a_whole_vocabulary(T, dtype):
    """50,304 entries, the large tiles among them, against float64 on the GPU."""
    import torch
    h, w, y, th, tw, ty = _inputs(T, 128, 50304, dtype, T)
    got = P.token_stats(th, tw, ty, 0.7, 8)
    logits = th.double() @ tw.double().T
    logp = torch.log_softmax(logits / 0.7, 1)
    tol = 2.0**-22 * float(logits.abs().max()) / 0.7 + 2.0**-21 + 900 * 2.0**-24
    ent = -(logp.exp() * logp).sum(1)
    assert ((got["entropy"] - ent).abs() <= 2 * tol * (1 + ent)).all()
    lp = torch.where(ty >= 0, logp.gather(1, ty.long().clamp(min=0)[:, None])[:, 0], 0.0)
    assert ((got["logprobs"] - lp).abs() <= 2 * tol).all()
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    assert (got["top_ids"] == order.indices[:, :8]).all()
    assert ((got["top_logprobs"] - logp.gather(1, order.indices[:, :8])).abs() <= 2 * tol).all()


def test_inputs_off_the_grid():
    """Any values: a logit is then off by at most (d + 2) 2^-24 of the sum of its products' magnitudes."""
    import torch
    g = np.random.default_rng(5)
    for dtype in ("fp32", "bf16", "fp16"):
        th, tw = (torch.from_numpy(g.normal(0, s, n)).to("cuda", _dt(dtype)) for s, n in ((1.0, (90, 640)), (0.05, (1200, 640))))
        h, w = th.double().cpu().numpy(), tw.double().cpu().numpy()
        y = g.integers(0, 1200, 90).astype(np.int32)
        want = oracle_stats(h, w, y, 0.7)
        got = P.token_stats(th, tw, y, 0.7)
        tol = 642 * 2.0**-24 * (np.abs(h) @ np.abs(w).T).max(1) / 0.7 + 1e-5
        assert (np.abs(got["logprobs"].cpu().numpy() - want["logprobs"]) <= 2 * tol).all()
        assert (np.abs(got["entropy"].cpu().numpy() - want["entropy"]) <= 2 * tol * (1 + want["entropy"])).all()


def test_equal_logits_go_to_the_lower_id():
    import torch
    T, d, V = 5, 64, 1000
    h, w = torch.ones(T, d, device="cuda", dtype=torch.bfloat16), torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    w[[700, 3, 130]] = 0.5
    w[[64, 999]] = 0.25
    got = P.token_stats(h, w, torch.zeros(T, dtype=torch.int32, device="cuda"), 1.0, 8)
    assert got["top_ids"].tolist() == [[3, 130, 700, 64, 999, 0, 1, 2]] * T
    neg = P.token_stats(-h, w * 0, [0] * T, 1.0, 3)  # sums of -0
    assert neg["top_ids"].tolist() == [[0, 1, 2]] * T
    assert torch.allclose(neg["entropy"], torch.full((T,), float(np.log(1000.0)), device="cuda"), rtol=1e-6)


@pytest.mark.parametrize("T,V,k", [(3, 5000, 20), (2, 5000, 50), (2, 300, 64), (2816, 50304, 8)])
def test_more_equal_logits_than_the_quick_way_holds(T, V, k):
    """All logits equal but one, last: its id first, then the lowest."""
    import torch
    h = torch.ones(T, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(V, 64, device="cuda", dtype=torch.bfloat16)
    w[V - 1] = 0.25
    got = P.token_stats(h, w, torch.full((T,), V - 1, dtype=torch.int32, device="cuda"), 0.7, k)
    want = torch.tensor([V - 1] + list(range(k - 1)), dtype=torch.int32, device="cuda")
    assert (got["top_ids"] == want).all()
    lse = np.log((V - 1) + np.exp(16 / 0.7))
    assert float((got["logprobs"] - (16 / 0.7 - lse)).abs().max()) <= 1e-4 and float((got["top_logprobs"][:, 1:] + lse).abs().max()) <= 1e-4


@pytest.mark.parametrize("k", [1, 8, 24, 40])
def test_rows_enough_for_part_of_the_logits_to_be_kept(k):
    """2,816 rows of 50,304 entries: after an eighth of the vocabulary only parts that can hold an alternative are stored."""
    import torch
    h, w, y, th, tw, ty = _inputs(2816, 64, 50304, "bf16", 5, lean=0.5)
    got = P.token_stats(th, tw, ty, 0.7, k)
    plain = P.token_stats(th, tw, ty, 0.7)
    logits = (th.double() @ tw.double().T)
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    assert (got["top_ids"] == order.indices[:, :k]).all()
    lse = torch.logsumexp(logits / 0.7, 1)
    tol = 2.0**-22 * float(logits.abs().max()) / 0.7 + 2.0**-21 + 900 * 2.0**-24
    assert ((got["top_logprobs"] - (order.values[:, :k] / 0.7 - lse[:, None])).abs() <= 2 * tol).all()
    for n in plain:
        assert (got[n] == plain[n]).all(), n


def test_one_sure_token_and_large_logits():
    """A token that has everything: its log-probability and the entropy are 0, not NaN; others' log-probabilities are their distance."""
    import torch
    h = torch.full((2, 64), 8.0, device="cuda", dtype=torch.float16)
    w = torch.zeros(300, 64, device="cuda", dtype=torch.float16)
    w[7] = 60.0
    got = P.token_stats(h, w, [7, 8], 0.5, 2)
    assert got["logprobs"].tolist() == [0.0, -61440.0] and got["entropy"].tolist() == [0.0, 0.0]
    assert got["top_ids"].tolist() == [[7, 0]] * 2 and got["top_logprobs"].tolist() == [[0.0, -61440.0]] * 2
    grad = P.token_stats_backward(h, w, [7, 7], got["lse"], got["entropy"], [1.0, 1.0], [1.0, 1.0], 0.5)
    assert (grad["d_hidden"] == 0).all() and (grad["d_weight"] == 0).all()


@pytest.mark.parametrize("dtype,V,k", [("fp16", 50304, 2), ("bf16", 700, 0), ("fp32", 700, 3)])
@pytest.mark.parametrize("T", [1, 300])
def test_a_token_with_nearly_everything_keeps_its_bits(T, dtype, V, k):
    """Row t's token is ahead by 4 + t % 12, so its log-probability is about -e^-16 at the least: held relative to itself, as is the
    entropy.  Beside the bars above (of values, where x is at most the row's spread of logits) the two sums of the entropy are of one
    sign, log1p adds 2^-22, and exp's argument, rounded three times, is off by 3 * 2^-24 x."""
    import torch
    g = np.random.default_rng(V + T)
    w = np.clip(np.round(g.normal(0, 0.04, (V, 64)) * 1024), -127, 127) / 1024
    w[:, 0] = 0
    y = g.integers(0, V, T).astype(np.int32)
    h = np.round(g.normal(0, 1, (T, 64)) * 16) / 16
    w2 = np.zeros((V, 32))  # 32 more features: a token has its own sign pattern there, a row its token's, times what leads by enough
    w2[:, :17] = 1 - 2.0 * ((np.arange(V)[:, None] >> np.arange(17)) & 1)
    want = []
    for t in range(T):
        z = h[t] @ w.T
        z0 = w2 @ w2[y[t]]  # 17, at others at most 15
        want.append(np.ceil(max(0.0, (4 + t % 12 + np.delete(z, y[t]).max() - z[y[t]]) / 2) * 8) / 8)
        assert (np.delete(z0, y[t]) <= 15).all()
    h2 = np.array(want)[:, None] * w2[y]
    h, w = np.concatenate([h, h2], 1), np.concatenate([w, w2], 1)
    dev = [torch.from_numpy(x).to("cuda", _dt(dtype)) for x in (h, w)]
    assert all((x.cpu().numpy() == e).all() for x, e in zip((dev[0].double(), dev[1].double()), (h, w)))
    got = P.token_stats(dev[0], dev[1], torch.from_numpy(y).cuda(), 1.0, k)
    z = h @ w.T
    x = z - z[np.arange(T), y][:, None]
    assert (np.sort(x, 1)[:, -2] <= -4).all()
    rest = np.where(x < 0, np.exp(x), 0).sum(1)
    lp = -np.log1p(rest)
    ent = -lp - np.where(x < 0, np.exp(x) * x, 0).sum(1) / (1 + rest)
    tol = 2.0**-22 * (2 + np.abs(x).max(1)) + 2.0**-21 + (100 + V / 64) * 2.0**-24
    for name, value in (("logprobs", lp), ("entropy", ent)):
        err = np.abs(got[name].cpu().numpy() - value) / np.abs(value)
        assert (err <= 2 * tol).all(), (name, err.max())
    if k:
        assert (got["top_ids"][:, 0].cpu().numpy() == y).all()
        assert (got["top_logprobs"][:, 0] == got["logprobs"]).all()


def test_rows_that_are_not_numbers_stay_alone():
    import torch
    h, w, y, th, tw, ty = _inputs(9, 64, 500, "bf16", 3)
    clean = P.token_stats(th, tw, ty, 0.7, 4)
    th[4, 5] = float("nan")
    got = P.token_stats(th, tw, ty, 0.7, 4)
    ok = torch.arange(9, device="cuda") != 4
    for n in clean:
        assert (got[n][ok] == clean[n][ok]).all(), n
    assert got["entropy"][4].isnan() and got["lse"][4].isnan()
    assert got["top_ids"][4].tolist() == [0, 1, 2, 3] and got["top_logprobs"][4].isnan().all()


def test_targets_outside_the_vocabulary_are_absent():
    import torch
    h, w, _, th, tw, _ = _inputs(4, 64, 50, "fp32", 1)
    y = np.array([-1, 50, 2**31 - 1, -(2**31)], np.int32)
    got = P.token_stats(th, tw, torch.from_numpy(y).cuda(), 0.7, 0)
    assert (got["logprobs"] == 0).all()
    grad = P.token_stats_backward(th, tw, torch.from_numpy(y).cuda(), got["lse"], None, torch.full((4,), 1e9, device="cuda"), None, 0.7)
    assert (grad["d_hidden"] == 0).all() and (grad["d_weight"] == 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_strided_rows_and_odd_bases(dtype):
    """Rows apart, a column offset that leaves 16 bytes, a transposed matrix: as the contiguous copy, bit for bit where no copy is made."""
    import torch
    T, d, V = 21, 64, 333
    h, w, y, th, tw, ty = _inputs(T, d, V, dtype, 8)
    want = P.token_stats(th, tw, ty, 0.7, 3)
    views = []
    for off in (0, 16, 3):
        wide_h, wide_w = (torch.full((n, d + e), 9.0, device="cuda", dtype=th.dtype) for n, e in ((T, 64), (V, 32)))
        wide_h[:, off:off + d], wide_w[:, off:off + d] = th, tw
        views.append((wide_h[:, off:off + d], wide_w[:, off:off + d]))
        got = P.token_stats(*views[-1], ty, 0.7, 3)
        for n in want:
            assert (got[n] == want[n]).all(), (off, n)
    got = P.token_stats(th.T.contiguous().T, tw.T.contiguous().T, ty, 0.7, 3)
    for n in want:
        assert (got[n] == want[n]).all(), n
    g = torch.randn(T, device="cuda")
    a = P.token_stats_backward(th, tw, ty, want["lse"], want["entropy"], g, 0.1 * g, 0.7)
    b = P.token_stats_backward(*views[1], ty, want["lse"], want["entropy"], g, 0.1 * g, 0.7)
    assert all((a[n] == b[n]).all() for n in a)


GRADS = [  # T, d, V, type, type of the gradients
    (1, 64, 100, "bf16", "bf16"), (1, 1, 1, "fp32", "fp32"), (3, 37, 77, "fp16", "fp16"), (6, 64, 64, "fp32", "fp32"),
    (70, 128, 513, "bf16", "bf16"), (129, 96, 1000, "fp32", "fp32"), (257, 192, 640, "fp16", "fp32"), (300, 72, 2050, "fp16", "fp16"),
    (1000, 64, 3001, "bf16", "fp32"), (64, 1030, 130, "bf16", "bf16"), (2100, 640, 4200, "bf16", "bf16"),
    (1, 64, 20011, "fp16", "fp16"), (33, 512, 40001, "bf16", "bf16"), (2, 128, 9999, "fp32", "fp32"), (40, 2048, 333, "fp32", "fp32"),
    (95, 160, 6001, "fp32", "fp32"),
]


def _check_grad(got, h, w, y, gl, ge, temp, dtype, gdtype, T):
    """dl is off by its rounding (half a step u) and by what its arithmetic loses: 2^-22 (|z| + 60) of the terms it is
    the difference of, and, since log p = z - lse and the entropy are differences of numbers of |z|'s size, which in fp32 are given
    to half an ulp each (2^-24 (|z| + |lse|), |lse| <= |z| + log V, and the bar of the forward call for the entropy), e p times what
    those are off absolutely, however small log p + entropy itself; the products add terms in fp32 (2^-24 of their magnitudes' sum each), and the result is rounded once more."""
    import torch
    dh, dw, dl = oracle_backward(h, w, y, gl, ge, temp)
    u = {"fp32": 0.0, "bf16": 2.0**-8, "fp16": 2.0**-11}
    z = h @ w.T / temp
    logp = z - z.max(1, keepdims=True)
    logp -= np.log(np.exp(logp).sum(1, keepdims=True))
    p = np.exp(logp)
    ent = -(p * logp).sum(1, keepdims=True)
    terms = p * (np.abs(gl)[:, None] * ((y >= 0) & (y < w.shape[0]))[:, None])
    if ge is not None:
        terms = terms + p * np.abs(ge)[:, None] * (np.abs(logp) + ent)
    off = 2.0**-23 * (2 * np.abs(z).max(1, keepdims=True) + np.log(len(w)))
    off = off + 2 * (2.0**-22 * np.abs(z).max(1, keepdims=True) + 2.0**-21 + (100 + len(w) / 64) * 2.0**-24) * (1 + ent)
    more = 0.0 if ge is None else p * np.abs(ge)[:, None] * off / temp
    err = more + u[dtype] * np.abs(dl) + (2.0**-22 * (np.abs(z).max() + 60)) * terms / temp + 2.0**-23 * np.abs(dl)
    if dtype == "fp16":
        err += 2.0**-25 * 2.0**-11 * np.abs(dl).max() * 64  # what falls below fp16's normal numbers once the largest is near 2^11
    for name, want, a, b, n in (("d_hidden", dh, err, np.abs(w), w.shape[0]), ("d_weight", dw, err.T, np.abs(h), T)):
        have = got[name].double().cpu().numpy()
        mags = (np.abs(dl) if name == "d_hidden" else np.abs(dl).T) @ b
        tol = a @ b + (n + 2) * 2.0**-24 * mags + u[gdtype] * np.abs(want) + (2.0**-25 if gdtype == "fp16" else 1e-37)
        tol += u[gdtype] * (a @ b)
        assert have.shape == want.shape and got[name].dtype == _dt(gdtype)
        assert (np.abs(have - want) <= tol).all(), (name, np.abs(have - want).max(), (np.abs(have - want) / tol).max())


@pytest.mark.parametrize("T,d,V,dtype,gdtype", GRADS)
def test_gradient_against_the_oracle(T, d, V, dtype, gdtype):
    h, w, y, th, tw, ty = _inputs(T, d, V, dtype, T + d + V)
    g = np.random.default_rng(T)
    gl, ge = g.normal(0, 1, T).astype(np.float32), g.normal(0, 0.2, T).astype(np.float32)
    s = P.token_stats(th, tw, ty, 0.7)
    got = P.token_stats_backward(th, tw, ty, s["lse"], s["entropy"], gl, ge, 0.7, grad_dtype=_dt(gdtype))
    _check_grad(got, h, w, y, gl, ge, 0.7, dtype, gdtype, T)
    got = P.token_stats_backward(th, tw, ty, s["lse"], None, gl, None, 0.7, grad_dtype=_dt(gdtype))
    _check_grad(got, h, w, y, gl, None, 0.7, dtype, gdtype, T)


@pytest.mark.parametrize("scale", [1e-7, 1e5])
def test_gradient_of_any_scale_in_half_precision(scale):
    """An unscaled loss's gradients (and very large ones) come out in fp32 as exactly as those of size one."""
    T, d, V = 60, 64, 400
    h, w, y, th, tw, ty = _inputs(T, d, V, "fp16", 4)
    g = np.random.default_rng(1)
    gl, ge = (scale * g.normal(0, 1, T)).astype(np.float32), (scale * g.normal(0, 0.1, T)).astype(np.float32)
    s = P.token_stats(th, tw, ty, 0.7)
    import torch
    got = P.token_stats_backward(th, tw, ty, s["lse"], s["entropy"], gl, ge, 0.7, grad_dtype=torch.float32)
    _check_grad(got, h, w, y, gl, ge, 0.7, "fp16", "fp32", T)


def test_gradient_over_several_chunks_of_rows():
    """16,500 rows: two chunks, whose sums meet in fp32; against float64 on the GPU, 2-norm: rounding of dl and of the result, half
    a step of 2^-8 each at most."""
    import torch
    for dtype, gdtype in (("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32")):
        T, d, V = 16500, 64, 300
        h, w, y, th, tw, ty = _inputs(T, d, V, dtype, 2)
        gl, ge = torch.randn(T, device="cuda"), 0.1 * torch.randn(T, device="cuda")
        s = P.token_stats(th, tw, ty, 0.7)
        got = P.token_stats_backward(th, tw, ty, s["lse"], s["entropy"], gl, ge, 0.7, grad_dtype=_dt(gdtype))
        logp = torch.log_softmax(th.double() @ tw.double().T / 0.7, 1)
        p = logp.exp()
        ent = -(p * logp).sum(1, keepdim=True)
        g = torch.where(ty >= 0, gl, 0.0).double()[:, None]
        dl = -p * (g + ge.double()[:, None] * (logp + ent))
        dl.scatter_add_(1, ty.long().clamp(min=0)[:, None], g)
        dl /= 0.7
        u = {"fp32": 1e-5, "bf16": 2.0**-8, "fp16": 2.0**-11}
        for n, want in (("d_hidden", dl @ tw.double()), ("d_weight", dl.T @ th.double())):
            assert float((got[n].double() - want).norm() / want.norm()) <= u[dtype] + u[gdtype] + 1e-5, (dtype, gdtype, n)


def test_offsets_beyond_32_bits():
    """8,300 rows of 262,144 entries: more logits, and more entries of dl, than 31 bits count; the first and the last of them.  The
    gradient's bars are those of the chunks' test."""
    import torch
    T, d, V = 8300, 64, 1 << 18
    h, w, y, th, tw, ty = _inputs(T, d, V, "bf16", 8)
    some = np.r_[0:5, T - 20:T]
    s = P.token_stats(th, tw, ty, 0.7, 3)
    _check({n: x[torch.from_numpy(some).cuda()] for n, x in s.items()}, h[some], w, y[some], 0.7, 3)
    gl, ge = torch.randn(T, device="cuda"), 0.1 * torch.randn(T, device="cuda")
    got = P.token_stats_backward(th, tw, ty, s["lse"], s["entropy"], gl, ge, 0.7)

    def dl(rows, cols):
        logp = th[rows].double() @ tw[cols].double().T / 0.7 - s["lse"][rows, None].double()
        g = torch.where(ty[rows] >= 0, gl[rows], 0.0).double()[:, None]
        p = logp.exp()
        own = ty[rows, None] == torch.arange(V, device="cuda")[cols]
        return (g * own - p * (g + ge[rows, None].double() * (logp + s["entropy"][rows, None].double()))) / 0.7

    everything = slice(0, None)
    for have, want in ((got["d_hidden"][-20:], dl(slice(T - 20, T), everything) @ tw.double()),
                       (got["d_hidden"][:5], dl(slice(0, 5), everything) @ tw.double()),
                       (got["d_weight"][-64:], dl(everything, slice(V - 64, V)).T @ th.double())):
        assert float((have.double() - want).norm() / want.norm()) <= 2 * 2.0**-8 + 1e-5


def test_gradient_matches_differences_of_the_forward_call():
    """fp32, through the library alone: the loss's change along a direction against the gradient."""
    import torch
    h, w, y, th, tw, ty = _inputs(12, 64, 90, "fp32", 6, lean=0.3)
    gl, ge = torch.randn(12, device="cuda"), torch.randn(12, device="cuda")
    s = P.token_stats(th, tw, ty, 0.7)
    got = P.token_stats_backward(th, tw, ty, s["lse"], s["entropy"], gl, ge, 0.7)

    def loss(a, b):
        o = P.token_stats(a, b, ty, 0.7)
        return float((gl.double() * o["logprobs"].double() + ge.double() * o["entropy"].double()).sum())

    eps = 2.0**-8
    for i, x, name in ((0, th, "d_hidden"), (1, tw, "d_weight")):
        v = torch.randn_like(x) / x.numel() ** 0.5
        up, down = [loss(*((x + q * eps * v, tw) if i == 0 else (th, x + q * eps * v))) for q in (1, -1)]
        along = float((got[name].double() * v.double()).sum())
        # third derivatives times eps^2 / 6, and 1e-6 of sums of order ten over 2 eps
        assert abs((up - down) / (2 * eps) - along) <= 2e-3 * (1 + abs(along))


def test_every_call_repeats_itself_and_reads_nothing_stale(monkeypatch):
    import torch
    monkeypatch.setattr(P.binding, "POISON", True)
    for T, d, V, dtype in ((45, 100, 1037, "bf16"), (300, 64, 50304, "fp16"), (33, 65, 70, "fp32")):
        h, w, y, th, tw, ty = _inputs(T, d, V, dtype, 11)
        gl = torch.randn(T, device="cuda")
        runs = []
        for _ in range(2):
            s = P.token_stats(th, tw, ty, 0.7, 6)
            runs.append({**s, **P.token_stats_backward(th, tw, ty, s["lse"], s["entropy"], gl, 0.1 * gl, 0.7)})
        assert all((runs[0][n] == runs[1][n]).all() for n in runs[0])
        assert all(torch.isfinite(v).all() for v in runs[0].values() if v.is_floating_point())


def test_no_rows():
    import torch
    h, w = torch.zeros(0, 64, device="cuda"), torch.ones(10, 64, device="cuda")
    out = P.token_stats(h, w, torch.zeros(0, dtype=torch.int32, device="cuda"), 0.7, 2)
    assert out["logprobs"].shape == (0,) and out["top_ids"].shape == (0, 2)
    z = torch.zeros(0, device="cuda")
    g = P.token_stats_backward(h, w, torch.zeros(0, dtype=torch.int32, device="cuda"), z, z, z, z)
    assert g["d_hidden"].shape == (0, 64) and (g["d_weight"] == 0).all() and g["d_weight"].shape == (10, 64)


def test_another_stream_and_a_captured_graph():
    import torch
    h, w, y, th, tw, ty = _inputs(70, 128, 2000, "bf16", 13)
    gl = torch.randn(70, device="cuda")

    def call():
        s = P.token_stats(th, tw, ty, 0.7, 5)
        return {**s, **P.token_stats_backward(th, tw, ty, s["lse"], s["entropy"], gl, 0.1 * gl, 0.7)}

    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all((got[n] == want[n]).all() for n in want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        kept = call()
    for k in range(3):  # replays between eager work, on inputs changed in place
        th.copy_(th.roll(k, 0))
        ty.copy_(ty.roll(k, 0))
        want = call()
        for v in kept.values():
            v.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert all((kept[n] == want[n]).all() for n in want), k


def test_gradients_of_two_graphs_do_not_meet():
    """Two captured calls of different inputs, replayed in turn: each has its own workspace."""
    import torch
    cases = [_inputs(40, 64, 700, "fp16", 20 + i)[3:] for i in range(2)]
    gl = torch.randn(40, device="cuda")

    def call(c):
        s = P.token_stats(*c, 0.7)
        return P.token_stats_backward(*c, s["lse"], s["entropy"], gl, gl, 0.7)

    want = [call(c) for c in cases]
    graphs = [torch.cuda.CUDAGraph() for _ in cases]
    kept = []
    torch.cuda.synchronize()
    for g, c in zip(graphs, cases):
        with torch.cuda.graph(g):
            kept.append(call(c))
    for _ in range(2):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for a, b in zip(kept, want):
        assert all((a[n] == b[n]).all() for n in b)


def test_refusals_of_the_binding():
    import torch
    h, w = torch.zeros(4, 64, device="cuda"), torch.zeros(9, 64, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: P.token_stats(h, w.half(), y), lambda: P.token_stats(h.double(), w.double(), y), lambda: P.token_stats(h, w[:, :32], y),
                lambda: P.token_stats(h, w, y[:3]), lambda: P.token_stats(h[0], w, y), lambda: P.token_stats(h, w, y, 0.7, 10),
                lambda: P.token_stats(h, w, y, 0.0), lambda: P.token_stats(h, w, y, 0.7, -1), lambda: P.token_stats(h, w[:0], y),
                lambda: P.token_stats_backward(h, w, y, y.float(), None, y.float(), y.float()),
                lambda: P.token_stats_backward(h, w, y, y.float()[:2], None, y.float()),
                lambda: P.token_stats_backward(h.half(), w.half(), y, y.float(), None, y.float(), grad_dtype=torch.bfloat16)):
        with pytest.raises(P.RlhfError):
            bad()
