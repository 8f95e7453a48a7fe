"""The 64-bit definitions of the training step's operators (oracle/step.py) against values worked by hand and, for the loss, against
differences: what the GPU tests compare with."""
import numpy as np
import pytest

from oracle import step as st


def test_logp_of_a_row_worked_by_hand():
    z = np.log(np.array([[1.0, 2.0, 5.0]]))         # probabilities 1/8, 2/8, 5/8
    assert np.allclose(st.policy_loss(z, [2])["logp"], np.log(5 / 8), rtol=1e-15)
    r = st.policy_loss(z, [1], old=[np.log(0.5)], adv=[3.0])       # ratio 1/2, advantage positive: not clipped
    assert np.allclose(r["loss"], -1.5) and np.allclose(r["grad"], [[-1.5 * -0.125, -1.5 * 0.75, -1.5 * -0.625]])
    r = st.policy_loss(z, [1], old=[np.log(0.5)], adv=[-3.0])      # ... negative: clipped at 0.8, no gradient
    assert np.allclose(r["loss"], 2.4) and not r["grad"].any() and r["sums"][3] == 1
    r = st.policy_loss(z, [1], old=[np.log(0.25)], ref=[np.log(0.5)], adv=[0.0], kl_coef=2.0)      # d = log 2
    assert np.allclose(r["loss"], 2.0 * (1.0 - np.log(2.0))) and np.allclose(r["grad"][0, 1], -2.0 * 0.75)


def test_rows_with_nothing_to_learn_from():
    z = np.array([[0.0, 1.0], [np.nan, 1.0], [0.0, 1.0], [-np.inf, -np.inf]])
    r = st.policy_loss(z, [0, 1, 2, 1], adv=np.ones(4), weight=[1.0, 0.0, 1.0, 1.0])
    assert r["sums"][4] == 1 and not r["grad"][1:].any() and not r["loss"][1:].any()


@pytest.mark.parametrize("c", [1.0, 1.4])
def test_gradient_against_differences(c):
    g = np.random.default_rng(5)
    rows, vocab, h = 6, 11, 1e-5
    z, t = g.normal(size=(rows, vocab)), g.integers(0, vocab, rows)
    kw = dict(adv=g.normal(size=rows), weight=np.array([1, 0.5, 2, 1, 1, 0]), scale=0.3, kl_coef=0.1, c=c)
    lp = st.policy_loss(z, t, c=c)["logp"]
    kw.update(old=lp - np.array([0.05, -0.5, 0.5, 0.1, -0.1, 0]), ref=lp + 0.2 * g.normal(size=rows))
    want = st.policy_loss(z, t, **kw)["grad"]
    for i in range(rows):
        for j in range(vocab):
            up, down = z.copy(), z.copy()
            up[i, j] += h
            down[i, j] -= h
            d = 0.3 * (st.policy_loss(up, t, **kw)["loss"].sum() - st.policy_loss(down, t, **kw)["loss"].sum()) / (2 * h)
            assert abs(d - want[i, j]) < 1e-8       # third derivatives below 10: h^2 * 10 / 6, and rounding 1e-16 / h


def test_norm_clip_and_update_worked_by_hand():
    assert st.grad_norm([[3.0], [], [4.0]], scale=0.5) == 2.5 and st.grad_norm([[3.0, -4.0]], "inf") == 4.0 and st.grad_norm([]) == 0.0
    assert st.clip_factor(0.5, 1.0, 0.25) == 0.25 and np.isclose(st.clip_factor(4.0, 1.0), 0.25)
    p, m, v = st.adamw([1.0], [2.0], [0.0], [0.0], 1, lr=0.1, beta1=0.9, beta2=0.99, eps=0.0, weight_decay=0.5)
    assert np.allclose([p[0], m[0], v[0]], [1.0 - 0.05 - 0.1, 0.2, 0.04])      # the first step is lr times the gradient's sign
