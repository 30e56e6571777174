"""The confidence split of a token whose retained routes weigh nothing (routing fills a token without a live
expert up with routes of weight 0): there is no proportion to spread by, and nothing is spread."""

import numpy as np
import pytest

from oracle import exfold_oracle as O
from oracle import operators_oracle as P

S = np.float32([[1, 2, 3], [4, 1, 5], [6, 7, 1]])
L = np.float32([[0, 0.5, 0.25], [0.75, 0, 0.5], [0.5, 0.25, 0]])


@pytest.mark.parametrize("opts", [dict(confidence=True), dict(confidence=True, renorm=True),
                                  dict(confidence=True, loss_cap=0.5, renorm=True), dict(renorm=True), {}])
def test_a_token_without_a_live_expert_folds_to_weights_of_zero(opts):
    l = np.array([[-np.inf, -np.inf, -np.inf], [0.0, -np.inf, -np.inf]])
    ids, w = P.route_experts(l, 2)
    assert ids.tolist() == [[0, 1], [0, 1]] and w.tolist() == [[0, 0], [1, 0]]
    keep = O.select_prefill(ids, w.astype(np.float32), np.ones(3, np.float32), 1)
    assert keep.tolist() == [[True, False], [True, False]]
    out_ids, out_w = O.fold_prefill_safeguarded(ids, w.astype(np.float32), keep, S, L, **opts)
    assert out_ids.tolist() == [[0], [0]] and out_w.tolist() == [[0.0], [1.0]]


def test_a_given_keep_row_of_weight_zero_gets_the_targets_share_only():
    # routes 0, 1, 2 of weights 0, 0, 1; the third is omitted: target 1 (loss 1/4), c = 3/4, S = 7
    ids, w = np.array([[0, 1, 2]], np.int32), np.float32([[0, 0, 1]])
    keep = np.array([[True, True, False]])
    _, fw = O.fold_prefill_safeguarded(ids, w, keep, S, L, confidence=True)
    assert fw.tolist() == [[0.0, 5.25]]
    _, fw = O.fold_prefill_safeguarded(ids, w, keep, S, L, confidence=True, renorm=True)
    assert fw.tolist() == [[0.0, 1.0]]
