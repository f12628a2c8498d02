"""The operators of an update together, as a training loop uses them: a policy's own hidden states and weights through the token
statistics, the gradient of a loss with an entropy bonus, and the optimizer steps.  Each link is checked against float64 on what
reached it."""
import numpy as np
import pytest

import paper_2403_17031_amd as P
from oracle.muon_oracle import muon_step
from synth import ModelConfig, make_weights

pytestmark = pytest.mark.gpu

CFG = ModelConfig(n_layers=2, d_model=128, n_heads=2, head_dim=64, rotary_dims=16, d_ff=512, vocab=1000, dtype="bf16", pad_id=999, eos_id=1)
MATRICES = ("w_qkv", "w_o", "w_fc1", "w_fc2")
TEMP = 0.7


@pytest.fixture(scope="module", autouse=True)
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.load_library()
    return P


def _batch(seed, B=6, Lq=20, N=12):
    g = np.random.default_rng(seed)
    L = Lq + N
    mask = np.ones((B, L), np.uint8)
    for b in range(B):
        mask[b, :g.integers(0, 8)] = 0
        mask[b, L - g.integers(0, N):] = 0
    tokens = np.where(mask == 1, g.integers(2, CFG.pad_id, (B, L)), CFG.pad_id).astype(np.int32)
    return tokens, mask, Lq


def _hidden(pol, x_last):
    """The final LayerNorm of the kept residual stream, as the heads see it (fp16)."""
    import torch
    g, b = (pol._dev[n].float() for n in ("lnf_g", "lnf_b"))
    return torch.nn.functional.layer_norm(x_last, (CFG.d_model,), g, b, CFG.ln_eps).half()


def _packed(tokens, mask):
    """Per packed row: the token it predicts (-1: none), and where that token lies in the padded batch."""
    y, where = [], []
    for b in range(tokens.shape[0]):
        cols = np.flatnonzero(mask[b])
        for c in cols:
            nxt = c + 1 in cols
            y.append(tokens[b, c + 1] if nxt else -1)
            where.append((b, c + 1 if nxt else -1))
    return np.array(y, np.int32), where


def test_statistics_of_a_policys_own_hidden_states():
    """Log-probabilities as score_sequences has them, and the first alternative is the argmax of the logits it shows."""
    import torch
    pol = P.Policy(CFG, make_weights(CFG, 3, variant="test"))
    tokens, mask, _ = _batch(1)
    x_keep, cu, _ = pol.forward_keep(tokens, mask)
    y, where = _packed(tokens, mask)
    T = len(y)
    s = P.token_stats(_hidden(pol, x_keep[-1][:T]), pol._dev["embed_out"].half(), y, TEMP, 5)
    lp, _ = pol.score_sequences(tokens, mask, TEMP)
    at = [i for i, w in enumerate(where) if w[1] >= 0]
    want = torch.stack([lp[where[i]] for i in at])
    # the same fp16 hidden states but for their last bit (another LayerNorm's order of sums): 2^-11 of a logit of about 10
    assert float((s["logprobs"][at] - want).abs().max()) <= 2e-2
    pairs = [(w[0], w[1] - 1) for w in where if w[1] >= 0]
    logits = pol.debug_logits_rows(tokens, mask, pairs)
    best = torch.gather(logits, 1, s["top_ids"][at][:, :1].long())[:, 0]
    assert float((logits.amax(1) - best).max()) <= 2e-2
    assert ((s["entropy"] >= 0) & (s["entropy"] <= np.log(CFG.vocab) + 1e-4)).all()
    pol.close()


def test_a_step_with_an_entropy_bonus():
    """PPO's loss with the entropies: head and hidden gradients against float64 autograd, then AdamW for the head and Muon for the
    layers' matrices; the policy that has taken the step scores as one that is made of the updated weights."""
    import torch
    w = make_weights(CFG, 4, variant="test")
    pol = P.Policy(CFG, w)
    tokens, mask, Lq = _batch(2)
    B, L = tokens.shape
    N = L - Lq
    T = int(mask.sum())
    y, where = _packed(tokens, mask)
    x_keep, cu, ptok = pol.forward_keep(tokens, mask)
    hidden, head = _hidden(pol, x_keep[-1][:T]), pol._dev["embed_out"].half()
    s = P.token_stats(hidden, head, y, TEMP)
    # the response's log-probabilities, padded, into the library's loss
    rows = [i for i, wh in enumerate(where) if wh[1] >= Lq]
    bt = np.array([(where[i][0], where[i][1] - Lq) for i in rows])
    new = torch.zeros(B, N, device="cuda")
    new[bt[:, 0], bt[:, 1]] = s["logprobs"][rows]
    kept = torch.from_numpy(mask[:, Lq:].sum(1).astype(np.int32)).cuda()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    adv, val, ret = (torch.randn(B, N, generator=g, device="cuda") for _ in range(3))
    stats, d_lp, d_v = P.ppo_loss(new, new + 0.01, adv, val, val, ret, kept)
    n = int(kept.sum())
    gl, ge = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    gl[rows] = d_lp[bt[:, 0], bt[:, 1]]
    ge[rows] = -0.05 / n
    grad = P.token_stats_backward(hidden, head, y, s["lse"], s["entropy"], gl, ge, TEMP, grad_dtype=torch.float32)
    # float64 autograd of sum gl * logprob + ge * entropy
    h64, w64 = hidden.double().requires_grad_(), head.double().requires_grad_()
    logp = torch.log_softmax(h64 @ w64.T / TEMP, 1)
    ty = torch.from_numpy(y).cuda().long()
    lp64 = torch.where(ty >= 0, logp.gather(1, ty.clamp(min=0)[:, None])[:, 0], 0.0)
    ent64 = -(logp.exp() * logp).sum(1)
    for name, want in (("entropy", ent64), ("logprobs", lp64)):
        assert float((s[name].double() - want.detach()).abs().max()) <= 1e-4, name
    (gl.double() * lp64 + ge.double() * ent64).sum().backward()
    for name, want in (("d_hidden", h64.grad), ("d_weight", w64.grad)):  # half a step of fp16 for dl, and the softmax's own 1e-5
        assert float((grad[name].double() - want).norm() / want.norm()) <= 2.0**-11 + 1e-4, name
    # the layers' gradients from the library's own backward pass, and both optimizers
    scale = 64.0 * n
    gv = torch.zeros(T, device="cuda")
    grads = pol.policy_backward(x_keep, cu, ptok, y, gl, gv, TEMP, grad_scale=scale)
    st = pol.train_state()
    names = [f"layers.{l}.{m}" for l in range(CFG.n_layers) for m in MATRICES]
    master = [st["master"][k] for k in names]
    before = [t.double().cpu().numpy() for t in master]
    moments = [torch.zeros_like(t) for t in master]
    P.muon_step(master, [grads[k] for k in names], moments, lr=1e-2, grad_scale=1 / scale, params_bf16=[pol._dev[k] for k in names])
    for k, p0, p1, m in zip(names, before, master, moments):
        want, want_m, _ = muon_step(p0, grads[k].double().cpu().numpy(), np.zeros_like(p0), 1e-2, grad_scale=1 / scale)
        decayed = p0 * (1 - 1e-2 * 0.01)
        off = np.linalg.norm(p1.double().cpu().numpy() - want) / np.linalg.norm(want - decayed)
        assert off <= 4e-3, (k, off)
        assert torch.equal(pol._dev[k], p1.to(torch.bfloat16))
    P.adamw_step(st["master"]["embed_out"], grad["d_weight"], st["exp_avg"]["embed_out"], st["exp_avg_sq"]["embed_out"], 1, lr=1e-3,
                 param_bf16=pol._dev["embed_out"])
    pol.refresh_weights()
    after = pol.score_sequences(tokens, mask, TEMP)
    made = P.Policy(CFG, {**w, **{k: pol._dev[k].float().cpu().numpy() for k in names + ["embed_out"]}})
    for a, b in zip(after, made.score_sequences(tokens, mask, TEMP)):
        assert torch.equal(a, b)
    made.close()
    pol.close()
