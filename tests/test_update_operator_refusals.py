"""What the token statistics and the orthogonalised update refuse, through the C ABI; needs no GPU: nothing is launched."""
import ctypes as C

import pytest

import paper_2403_17031_amd as P
from paper_2403_17031_amd.binding import _MuonTensor

OK, EINVAL, ENOMEM, EUNSUPPORTED = 0, -1, -2, -4
PTR = 1 << 20  # stands for a device address; no refused call looks at what is there


@pytest.fixture(scope="module")
def lib():
    return P.load_library()


def _stats(lib, **over):
    a = dict(h=PTR, ldh=64, w=PTR, ldw=64, y=PTR, T=3, d=64, V=100, dtype=1, temp=0.7, k=2, lp=PTR, ent=PTR, lse=PTR, ids=PTR,
             tlp=PTR, ws=PTR, n=1 << 40)
    a.update(over)
    return lib.rlhf_token_stats(a["h"], a["ldh"], a["w"], a["ldw"], a["y"], a["T"], a["d"], a["V"], a["dtype"], a["temp"], a["k"],
                                a["lp"], a["ent"], a["lse"], a["ids"], a["tlp"], a["ws"], a["n"], None)


@pytest.mark.parametrize("over,rc", [
    (dict(T=0), EINVAL), (dict(d=0), EINVAL), (dict(V=-1), EINVAL), (dict(dtype=3), EUNSUPPORTED), (dict(ldh=63), EINVAL),
    (dict(ldw=63), EINVAL), (dict(V=262145, k=0), EUNSUPPORTED), (dict(k=-1), EINVAL), (dict(k=101), EINVAL),
    (dict(k=65), EUNSUPPORTED), (dict(h=None), EINVAL), (dict(w=None), EINVAL), (dict(y=None), EINVAL), (dict(lp=None), EINVAL),
    (dict(ent=None), EINVAL), (dict(lse=None), EINVAL), (dict(ids=None), EINVAL), (dict(tlp=None), EINVAL), (dict(ws=None), EINVAL),
    (dict(temp=0.0), EINVAL), (dict(temp=-1.0), EINVAL), (dict(temp=float("nan")), EINVAL), (dict(temp=float("inf")), EINVAL),
    (dict(h=PTR + 8), EINVAL), (dict(w=PTR + 2), EINVAL), (dict(ws=PTR + 4), EINVAL), (dict(n=0), ENOMEM),
    (dict(temp=1e-39), EINVAL), (dict(ldh=1 << 23), EUNSUPPORTED), (dict(T=(1 << 26) + 1), EUNSUPPORTED),
])
def test_token_stats_refusals(lib, over, rc):
    assert _stats(lib, **over) == rc and lib.rlhf_last_error()


def test_the_reported_workspace_is_the_least(lib):
    out = C.c_size_t()
    for T, d, V, ld, dtype, k in ((1, 64, 100, 64, 1, 0), (5000, 2560, 50304, 2560, 1, 8), (77, 37, 1000, 41, 2, 3), (9, 96, 640, 96, 0, 64)):
        assert lib.rlhf_token_stats_workspace_bytes(T, d, V, ld, ld, dtype, k, C.byref(out)) == OK
        assert _stats(lib, T=T, d=d, V=V, ldh=ld, ldw=ld, dtype=dtype, k=k, n=out.value - 1) == ENOMEM
    # without alternatives no logits are kept; a width that the products do not divide costs copies of both matrices
    sizes = []
    for d, k in ((2560, 0), (2560, 1), (2561, 0)):
        assert lib.rlhf_token_stats_workspace_bytes(4096, d, 50304, d, d, 1, k, C.byref(out)) == OK
        sizes.append(out.value)
    assert sizes[1] - sizes[0] >= 4096 * 50304 * 4 and sizes[2] - sizes[0] >= (4096 + 50304) * 2561 * 2
    assert lib.rlhf_token_stats_workspace_bytes(1, 1, 1, 1, 1, 1, 0, None) == EINVAL


def _grad(lib, **over):
    a = dict(h=PTR, ldh=64, w=PTR, ldw=64, y=PTR, lse=PTR, ent=PTR, g=PTR, e=PTR, T=3, d=64, V=100, dtype=1, temp=0.7, gdt=1, dh=PTR,
             dw=PTR, ws=PTR, n=1 << 40)
    a.update(over)
    return lib.rlhf_token_stats_backward(a["h"], a["ldh"], a["w"], a["ldw"], a["y"], a["lse"], a["ent"], a["g"], a["e"], a["T"], a["d"],
                                         a["V"], a["dtype"], a["temp"], a["gdt"], a["dh"], a["dw"], a["ws"], a["n"], None)


@pytest.mark.parametrize("over,rc", [
    (dict(T=0), EINVAL), (dict(dtype=-1), EUNSUPPORTED), (dict(gdt=2), EUNSUPPORTED), (dict(dtype=0, gdt=1), EUNSUPPORTED),
    (dict(lse=None), EINVAL), (dict(ent=None), EINVAL), (dict(g=None), EINVAL), (dict(dh=None), EINVAL), (dict(dw=None), EINVAL),
    (dict(temp=0.0), EINVAL), (dict(h=PTR + 8), EINVAL), (dict(n=0), ENOMEM), (dict(ldw=1), EINVAL),
])
def test_token_stats_backward_refusals(lib, over, rc):
    assert _grad(lib, **over) == rc and lib.rlhf_last_error()


def _orth(lib, **over):
    a = dict(x=PTR, dtype=0, batch=2, rows=5, cols=7, steps=5, eps=1e-7, out=PTR, ws=PTR, n=1 << 40)
    a.update(over)
    return lib.rlhf_orthogonalize(a["x"], a["dtype"], a["batch"], a["rows"], a["cols"], a["steps"], a["eps"], a["out"], a["ws"], a["n"], None)


@pytest.mark.parametrize("over,rc", [
    (dict(batch=0), EINVAL), (dict(rows=0), EINVAL), (dict(cols=-3), EINVAL), (dict(x=None), EINVAL), (dict(out=None), EINVAL),
    (dict(ws=None), EINVAL), (dict(dtype=2), EUNSUPPORTED), (dict(steps=0), EINVAL), (dict(steps=17), EINVAL), (dict(eps=0.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(n=0), ENOMEM), (dict(rows=32769, cols=32769), EUNSUPPORTED),
    (dict(rows=(1 << 20) + 1, cols=1), EUNSUPPORTED), (dict(rows=1 << 17, cols=1 << 14), EUNSUPPORTED), (dict(x=PTR + 2), EINVAL), (dict(ws=PTR + 8), EINVAL),
])
def test_orthogonalize_refusals(lib, over, rc):
    assert _orth(lib, **over) == rc and lib.rlhf_last_error()


def _muon(lib, tensors, count=None, **over):
    a = dict(lr=1e-3, mu=0.95, nest=1, wd=0.0, rms=0.2, steps=5, eps=1e-7, gs=1.0, ws=PTR, n=1 << 40)
    a.update(over)
    ts = (_MuonTensor * max(len(tensors), 1))(*tensors)
    return lib.rlhf_muon_step(ts, len(tensors) if count is None else count, a["lr"], a["mu"], a["nest"], a["wd"], a["rms"], a["steps"],
                              a["eps"], a["gs"], a["ws"], a["n"], None)


def _t(i=0, rows=5, cols=7, **over):
    a = dict(param=PTR * (3 * i + 1), grad=PTR * (3 * i + 2), momentum=PTR * (3 * i + 3), param_bf16=None)
    a.update(over)
    return _MuonTensor(a["param"], a["grad"], a["momentum"], a["param_bf16"], rows, cols)


@pytest.mark.parametrize("tensor", [_t(param=None), _t(grad=None), _t(momentum=None), _t(rows=-1), _t(param=PTR + 2), _t(param_bf16=PTR + 1)])
def test_muon_refuses_a_tensor(lib, tensor):
    assert _muon(lib, [tensor]) == EINVAL and lib.rlhf_last_error()


@pytest.mark.parametrize("over,rc", [
    (dict(mu=1.0), EINVAL), (dict(mu=-0.1), EINVAL), (dict(lr=-1.0), EINVAL), (dict(lr=float("nan")), EINVAL), (dict(wd=-1.0), EINVAL),
    (dict(rms=float("inf")), EINVAL), (dict(gs=float("nan")), EINVAL), (dict(steps=0), EINVAL), (dict(eps=0.0), EINVAL), (dict(n=0), ENOMEM),
    (dict(ws=None), EINVAL), (dict(ws=PTR + 4), EINVAL), (dict(count=-1), EINVAL),
])
def test_muon_refusals(lib, over, rc):
    assert _muon(lib, [_t()], **over) == rc and lib.rlhf_last_error()


def test_muon_refuses_an_array_twice(lib):
    assert _muon(lib, [_t(0), _t(1, param=PTR)]) == EINVAL
    assert _muon(lib, [_t(0), _t(1), _t(2, momentum=PTR * 3)]) == EINVAL


def test_nothing_to_do_is_no_error(lib):
    assert _muon(lib, [], ws=None, n=0) == OK
    assert _muon(lib, [_t(0, rows=0), _t(1, cols=0, param=None)], ws=None, n=0) == OK


def test_workspaces_of_many_matrices_stay_bounded(lib):
    """Matrices go together up to 2^28 elements, so the workspace of many is that of the largest group."""
    out = C.c_size_t()
    sizes = []
    for layers in (1, 8, 32):
        ts = (_MuonTensor * (2 * layers))(*[_t(i, rows=10240 >> (2 * (i & 1)), cols=2560) for i in range(2 * layers)])
        assert lib.rlhf_muon_workspace_bytes(ts, len(ts), C.byref(out)) == OK
        sizes.append(out.value)
    assert sizes[0] < sizes[1] == sizes[2] < 4 << 30
    one = C.c_size_t()
    assert lib.rlhf_orthogonalize_workspace_bytes(1, 77, 1000, C.byref(one)) == OK
    assert lib.rlhf_orthogonalize_workspace_bytes(1000, 77, 1000, C.byref(out)) == OK and one.value < out.value < 50 * one.value


def test_the_binding_refuses_tensors_off_the_gpu():
    import torch
    x = torch.zeros(4, 4)
    with pytest.raises(P.RlhfError, match="CUDA"):
        P.token_stats(x, x, [0, 0, 0, 0])
    with pytest.raises(P.RlhfError, match="CUDA"):
        P.token_stats_backward(x, x, [0] * 4, x[0], x[0], x[0])
    with pytest.raises(P.RlhfError, match="CUDA"):
        P.orthogonalize(x)
    with pytest.raises(P.RlhfError, match="CUDA"):
        P.muon_step([x], [x], [x])
    with pytest.raises(P.RlhfError, match="length"):
        P.muon_step([x], [], [x])
