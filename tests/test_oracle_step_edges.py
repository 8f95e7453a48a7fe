"""The 64-bit definition of the policy loss where a token is banned: what the GPU tests of it compare with."""
import numpy as np

from oracle import step as st

Z = np.array([[np.log(1.0), np.log(2.0), np.log(5.0), -np.inf]])


def test_a_token_that_the_policy_bans():
    r = st.policy_loss(Z, [3], old=[-1.0], ref=[-1.0], adv=[2.0])
    assert r["logp"][0] == -np.inf and r["loss"][0] == 0.0 and not r["grad"].any() and r["sums"][2] == np.inf
    assert st.policy_loss(Z, [3], ref=[-1.0], adv=[2.0], kl_coef=0.5)["loss"][0] == np.inf


def test_a_token_that_the_reference_bans():
    lp = np.log(2.0 / 8.0)
    plain = st.policy_loss(Z, [1], old=[lp], adv=[2.0])
    r = st.policy_loss(Z, [1], old=[lp], ref=[-np.inf], adv=[2.0])
    assert r["loss"][0] == plain["loss"][0] == -2.0 and np.array_equal(r["grad"], plain["grad"]) and r["sums"][2] == np.inf
    r = st.policy_loss(Z, [1], old=[lp], ref=[-np.inf], adv=[2.0], kl_coef=0.5)      # exp(d) - 1 = -1: the slope is -2 + 0.5
    assert r["loss"][0] == np.inf and np.allclose(r["grad"], -1.5 * np.array([[-0.125, 0.75, -0.625, 0.0]]))
