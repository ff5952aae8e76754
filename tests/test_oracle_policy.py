"""Pins of the oracle's policy update: its gradient against differences of its own loss, its terms against closed forms, and torch's
float64 differentiation of the formulas as an independent witness."""
import numpy as np
import pytest
import torch

import oracle


def _case(B, G, T, A, seed):
    rng = np.random.default_rng(seed)
    x = 1.5 * rng.standard_normal((B, G, T, A))
    ids = rng.integers(0, A, (B, G, T))
    old = np.array([oracle._log_softmax(x[i], 1.0)[ids[i]] for i in np.ndindex(B, G, T)]).reshape(B, G, T)
    old = old + rng.choice((-0.4, -0.1, 0.1, 0.4), (B, G, T))            # on both sides of both bounds, not near them
    return x, ids, rng.standard_normal((B, G, T)), old, old + 0.3 * rng.standard_normal((B, G, T)), x + 0.5 * rng.standard_normal(x.shape)


@pytest.mark.parametrize("kl", ["none", "logp", "logits"])
@pytest.mark.parametrize("mean", ["steps", "schedules"])
def test_gradient_against_differences(kl, mean):
    x, ids, adv, old, ref, ref_x = _case(2, 2, 3, 5, 1)
    eff = np.array([[1, 1, 0], [0, 1, 0]])
    kw = dict(old_logp=old, eff=eff, clip=(0.2, 0.28), entropy_coef=0.05, temperature=1.0, scale=0.5, mean=mean,
              kl_coef=0.0 if kl == "none" else 0.1, ref_logp=ref if kl == "logp" else None, ref_logits=ref_x if kl == "logits" else None)
    grad = oracle.policy_loss(x, ids, adv, **kw)["grad"]
    h = 1e-5
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        d = (oracle.policy_loss(up, ids, adv, **kw)["loss"] - oracle.policy_loss(down, ids, adv, **kw)["loss"]) / (2 * h)
        assert abs(d - grad[i]) < 1e-8                                   # h^2 = 1e-10 times third derivatives below 10; 1e-16 / h


@pytest.mark.parametrize("temperature", [1.0, 1.3])
@pytest.mark.parametrize("kl", ["none", "logp", "logits"])
def test_against_differentiation_by_torch(kl, temperature):
    x, ids, adv, old, ref, ref_x = _case(2, 3, 4, 7, 2)
    ref_x[..., 2] = x[..., 2] = -np.inf
    ids[ids == 2] = 0
    kw = dict(clip=(0.2, 0.28), entropy_coef=0.05, temperature=temperature, scale=0.5, kl_coef=0.0 if kl == "none" else 0.1)
    got = oracle.policy_loss(x, ids, adv, old_logp=old, ref_logp=ref if kl == "logp" else None, ref_logits=ref_x if kl == "logits" else None, **kw)
    t = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(t / temperature, -1)
    fin = lp.masked_fill(lp == -np.inf, 0.0)
    logp = lp.gather(-1, torch.tensor(ids)[..., None])[..., 0]
    ratio, a = (logp - torch.tensor(old)).exp(), torch.tensor(adv)
    loss = -torch.min(ratio * a, ratio.clamp(0.8, 1.28) * a) + 0.05 * (lp.exp() * fin).sum(-1)
    if kl == "logp":
        u = torch.tensor(ref) - logp
        loss = loss + 0.1 * (u.exp() - u - 1)
    if kl == "logits":
        lq = torch.log_softmax(torch.tensor(ref_x) / temperature, -1)
        loss = loss + 0.1 * (lp.exp() * (fin - lq.masked_fill(lq == -np.inf, 0.0))).sum(-1)
    loss = 0.5 * loss.mean()
    loss.backward()
    assert abs(float(loss.detach()) - got["loss"]) < 1e-12
    np.testing.assert_allclose(got["grad"], t.grad.numpy(), rtol=0, atol=1e-14)


def test_terms_in_closed_form():
    x = np.zeros((1, 1, 2, 4))
    r = oracle.policy_loss(x, np.zeros((1, 1, 2), int), np.array([[[1.0, -2.0]]]), entropy_coef=1.0, ref_logits=x + 3.0, kl_coef=1.0)
    np.testing.assert_allclose(r["stats"], [0.5, 0.0, np.log(4.0), 0.0], atol=1e-15)        # ratio 1: minus the mean advantage
    np.testing.assert_allclose(r["logp"], -np.log(4.0))
    np.testing.assert_allclose(r["grad"][0, 0, 0], 0.5 * np.array([-0.75, 0.25, 0.25, 0.25]), atol=1e-15)
    # both bounds: only the pessimistic side is cut
    for a, d, held in ((1.0, 0.5, True), (1.0, -0.5, False), (-1.0, 0.5, False), (-1.0, -0.5, True)):
        r = oracle.policy_loss(x[:, :, :1], np.zeros((1, 1, 1), int), np.full((1, 1, 1), a), old_logp=np.full((1, 1, 1), -np.log(4.0) - d))
        assert r["stats"][3] == held and (np.abs(r["grad"]).max() == 0.0) == held


def test_steps_and_schedules_weigh_ragged_inputs_differently():
    x, ids, adv, *_ = _case(2, 1, 4, 3, 5)
    eff = np.array([[1, 1, 1, 1], [1, 0, 0, 0]])
    steps, sched = (oracle.policy_loss(x, ids, adv, eff=eff, mean=m)["stats"][0] for m in ("steps", "schedules"))
    assert np.isclose(steps, -(adv[0, 0].sum() + adv[1, 0, 0]) / 5)
    assert np.isclose(sched, -(adv[0, 0].mean() + adv[1, 0, 0]) / 2)
    none = oracle.policy_loss(x, ids, adv, eff=np.zeros((2, 4)))
    assert none["loss"] == 0.0 and not none["grad"].any()


def test_clip_and_update_against_torch():
    rng = np.random.default_rng(6)
    ps = [torch.tensor(rng.standard_normal(s), requires_grad=True) for s in ((3, 4), (5,))]
    opt = torch.optim.AdamW(ps, lr=1e-2, betas=(0.9, 0.99), eps=1e-7, weight_decay=0.1)
    mine = [[p.detach().numpy().copy(), np.zeros(p.shape), np.zeros(p.shape)] for p in ps]
    for t in range(1, 5):
        grads = [rng.standard_normal(p.shape) for p in ps]
        for p, g in zip(ps, grads):
            p.grad = torch.tensor(g)
        norm, coef, _ = oracle.grad_clip(grads, 0.7)
        total = torch.nn.utils.clip_grad_norm_(ps, 0.7)
        assert np.isclose(norm, float(total), rtol=1e-14)
        opt.step()
        for i, (state, g) in enumerate(zip(mine, grads)):
            mine[i] = list(oracle.adamw_step(state[0], g, state[1], state[2], t, 1e-2, (0.9, 0.99), 1e-7, 0.1, coef))
            np.testing.assert_allclose(mine[i][0], ps[i].detach().numpy(), rtol=0, atol=1e-14)
