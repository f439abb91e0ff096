"""The decoding oracle is what its definitions say: softmax over the joined keys, weights that sum to the number of rows, drafting
that leaves the target's distribution as it is, caches that keep the largest weights."""
import numpy as np
import pytest

from oracle import attention_oracle as orc
from oracle import decoding_oracle as dec


@pytest.mark.parametrize("causal", [False, True])
def test_prefix_is_a_cache_that_begins_with_it(causal):
    r = np.random.default_rng(1)
    B, nq, hq, hkv, d, n_p, cap, lens = 3, 2, 4, 2, 8, 5, 7, np.array([7, 2, 4])
    Q, Kp, Vp = r.normal(size=(B, nq, hq, d)), r.normal(size=(n_p, hkv, d)), r.normal(size=(n_p, hkv, d))
    K, V = r.normal(size=(B, cap, hkv, d)), r.normal(size=(B, cap, hkv, d))
    O, L, A, M = dec.prefix_forward(Q, Kp, Vp, K, V, lens, 0.3, causal)
    join = lambda p, x: np.stack([np.concatenate([p, x[b]]) for b in range(B)])  # noqa: E731
    eO, eL = orc.kvcache_forward(Q, join(Kp, K), join(Vp, V), 0.3, causal, lens + n_p)
    np.testing.assert_allclose(O, eO, atol=1e-12)
    np.testing.assert_allclose(L, eL, atol=1e-12)
    assert (A >= np.abs(O) - 1e-12).all() and (M > 0).all()


def test_weights_of_a_row_sum_to_one():
    r = np.random.default_rng(2)
    Q, K = r.normal(size=(1, 3, 4, 8)), r.normal(size=(1, 6, 2, 8))
    _, L, _, _ = dec.prefix_forward(Q, np.zeros((0, 2, 8)), np.zeros((0, 2, 8)), K, K, [6], 0.3, True)
    (w,), _ = dec.key_weights(Q, K, L, [6], 0.3, True)
    np.testing.assert_allclose(w.sum(1), 3 * 2)  # three queries, two heads a group
    (w,), _ = dec.key_weights(Q, K, L, [6], 0.3, True, queries=[1])
    np.testing.assert_allclose(w.sum(1), 2)
    assert (w[:, 4:] == 0).all()


def test_kept_slots():
    w = np.array([5.0, 1.0, 1.0, np.nan, 0.0, 9.0, 2.0])
    pos = np.array([0, 6, 2, 3, 4, 5, 1])
    assert dec.kept_slots(w, pos, 7, 7, 0, 0).tolist() == list(range(7))
    assert dec.kept_slots(w, pos, 7, 3, 0, 0).tolist() == [0, 5, 6]
    assert dec.kept_slots(w, pos, 7, 4, 0, 0).tolist() == [0, 1, 5, 6]  # the lower of the equals
    assert dec.kept_slots(w, pos, 7, 3, 0, 1).tolist() == [0, 1, 5]  # position 6 is the newest
    assert dec.kept_slots(w, pos, 7, 3, 1, 2).tolist() == [0, 1, 5]
    assert dec.kept_slots(w, pos, 5, 4, 0, 0).tolist() == [0, 1, 2, 4]  # the NaN goes first


@pytest.mark.parametrize("certain", [False, True])
def test_drafting_leaves_the_distribution_as_it_is(certain):
    """The first token, over a grid of both random numbers and drafts in proportion to q, is distributed as p_0."""
    p = np.array([0.5, 0.2, 0.3, 0.0])
    q = np.array([0.25, 0.5, 0.0, 0.25])
    n = 100
    grid = (np.arange(n) + 0.5) / n
    count = np.zeros(4)
    for x in range(4):
        share = (1.0 if x == 1 else 0.0) if certain else q[x]
        if share == 0:
            continue
        u = np.stack(np.meshgrid(grid, grid), -1).reshape(-1, 2)
        t, _, _ = dec.verify(np.full((len(u), 1), x), None if certain else np.tile(q, (len(u), 1, 1)), np.tile(p, (len(u), 2, 1)), u)
        count += share * np.bincount(t[:, 0], minlength=4) / len(u)
    np.testing.assert_allclose(count, p, atol=2 / n)


def test_verify_edges():
    p = np.array([[[0.0, 1.0, 0.0], [0.5, 0.0, 0.5]]])
    q = np.array([[[0.0, 1.0, 0.0]]])
    assert dec.verify(np.array([[1]]), q, p, np.array([[0.9, 0.0]]))[0].tolist() == [[1, 0]]
    assert dec.verify(np.array([[1]]), q, p, np.array([[0.9, 0.5]]))[0].tolist() == [[1, 2]]  # the sum has to exceed
    assert dec.verify(np.array([[-1]]), q, p, np.array([[0.9, 0.5]]))[0].tolist() == [[1, -1]]
    assert dec.verify(np.array([[0]]), None, p, np.array([[0.0, 0.5]]))[0].tolist() == [[1, -1]]
    assert dec.verify(np.array([[1]]), np.ones((1, 1, 3)), 0 * p, np.array([[0.9, 0.5]]))[0].tolist() == [[-1, -1]]
    lp = np.where(p > 0, np.log(np.maximum(p, 1e-300)), -np.inf)
    assert dec.verify(np.array([[1]]), q, lp, np.array([[0.9, 0.6]]), logits=True)[0].tolist() == [[1, 2]]
