"""The value of the distillation loss, lists that name an id more than once among them: the oracle against the library's divergence over the whole vocabulary."""
import numpy as np
import pytest
import torch

from oracle import pp_oracle as O


def whole_rows(x, w, ids, u, tau):
    """Teacher's and student's log probabilities over the vocabulary, the teacher's entries of one id added up."""
    z = torch.tensor(x @ w.T)
    full = torch.full_like(z, -torch.inf)
    for t in range(len(ids)):
        for i, v in zip(ids[t], u[t]):
            if 0 <= i < z.shape[1]:
                full[t, i] = torch.logaddexp(full[t, i], torch.tensor(v / tau))
    return torch.log_softmax(full, 1), torch.log_softmax(z / tau, 1)


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_a_list_of_different_ids_has_the_divergence_over_the_vocabulary(tau):
    """The whole value, entropy included: 1 to 9 of 23 words listed, the others of probability 0."""
    r = np.random.default_rng(3)
    x, w, u = r.normal(size=(40, 5)), r.normal(size=(23, 5)), 2 * r.normal(size=(40, 9))
    ids = np.stack([r.permutation(23)[:9] for _ in range(40)])
    ids[np.arange(9)[None] >= r.integers(1, 10, (40, 1))] = -1
    logq, logp = whole_rows(x, w, ids, u, tau)
    want = tau ** 2 * torch.nn.functional.kl_div(logp, logq, reduction="none", log_target=True).nan_to_num(0.0).sum(1)
    got = O.head_loss(x, w, None, None, ids, u, tau, 1.0)["row_loss"]
    np.testing.assert_allclose(got, want.numpy(), rtol=1e-11, atol=1e-13)
    assert got.min() >= 0


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_a_repeated_id_lowers_the_value_by_its_split_and_changes_no_gradient(tau):
    r = np.random.default_rng(4)
    x, w = r.normal(size=(30, 5)), r.normal(size=(11, 5))
    ids, u = r.integers(0, 11, (30, 8)), 2 * r.normal(size=(30, 8))
    logq, logp = whole_rows(x, w, ids, u, tau)
    want = tau ** 2 * torch.nn.functional.kl_div(logp, logq, reduction="none", log_target=True).nan_to_num(0.0).sum(1).numpy()
    ref = O.head_loss(x, w, None, None, ids, u, tau, 1.0)
    q = torch.softmax(torch.tensor(u) / tau, 1).numpy()
    together = np.where(ids[:, :, None] == ids[:, None, :], q[:, None, :], 0.0).sum(2)
    split = tau ** 2 * (q * np.log(together / q)).sum(1)
    assert split.max() > 0.1
    np.testing.assert_allclose(ref["row_loss"] + split, want, rtol=1e-11, atol=1e-12)
    # the same teacher with its entries merged: the same gradients
    merged = O.head_loss(x, w, None, None, np.tile(np.arange(11), (30, 1)), tau * logq.numpy(), tau, 1.0)
    np.testing.assert_allclose(merged["row_loss"], want, rtol=1e-11, atol=1e-12)
    np.testing.assert_allclose(merged["dx"], ref["dx"], rtol=1e-10, atol=1e-14)
    np.testing.assert_allclose(merged["dw"], ref["dw"], rtol=1e-10, atol=1e-14)


def test_a_word_in_two_halves_has_a_negative_value():
    """log 1/2 - log p for two equal entries of a word that the student is sure of."""
    got = O.head_loss([[1.0]], [[10.0], [0.0]], None, None, np.array([[0, 0]]), np.zeros((1, 2)), 1.0, 1.0)["row_loss"][0]
    assert got == pytest.approx(np.log(0.5) + np.log1p(np.exp(-10.0)), abs=1e-14)
