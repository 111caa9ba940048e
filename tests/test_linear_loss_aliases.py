"""Outputs of the output layer's losses and of the top logits over scale words, and scale words over arrays, are refused (no GPU
needed: a call that fails validation launches nothing)."""
import pytest

import paper_2407_17353_b200 as sc
from test_linear_loss_refusals import B, F, IDS, LOSS, LSE, MB, MEAN, R, ce, ce_bwd, kd, kd_bwd
from test_operator_refusals import ALIAS, arr


@pytest.mark.parametrize("call", [ce, kd])
def test_forward_outputs_over_scale_words(call):
    for at, out in ((64, "mean"), (LOSS + 12, None), (LSE, None), (MEAN, None)):
        extra = {out: at} if out else {}
        assert call(H=arr(1, B, (4, 64), scale=at), **extra) == ALIAS
        assert call(W=arr(2, B, (100, 64), scale=at), **extra) == ALIAS
    if call is kd:
        assert call(T=arr(3, F, (4, 8), scale=LSE + 4)) == ALIAS


@pytest.mark.parametrize("call", [ce_bwd, kd_bwd])
def test_gradients_scale_words_over_arrays(call):
    out = lambda at: (arr(14, B, (4, 64), scale=at), arr(15, B, (100, 64), scale=at))  # noqa: E731
    for at in (MB + 64, 2 * MB + 100 * 128 - 4, IDS + 8, LSE + 12, 13 * MB + 4, 14 * MB + 4, 15 * MB + 4):   # H, W, ids, lse, grad, dH, dW
        dH, dW = out(at)
        assert call(dH=dH) == ALIAS and call(dW=dW) == ALIAS
    for which, a in (("H", arr(1, B, (4, 64), scale=14 * MB + 8)), ("W", arr(2, B, (100, 64), scale=15 * MB + 8)), ("grad", arr(13, F, (4,), scale=15 * MB))):
        assert call(**{which: a}) == ALIAS
    if call is kd_bwd:
        assert call(T=arr(3, F, (4, 8), scale=14 * MB)) == ALIAS and call(dH=out(3 * MB + 16)[0]) == ALIAS
        assert call(tl=12 * MB, dH=out(12 * MB + 4)[0]) == ALIAS


def test_a_word_between_rows_is_no_overlap():
    """Not refused as an alias (what comes back is the missing workspace)."""
    H = arr(1, B, (4, 64), (128, 1))
    assert ce_bwd(H=H, dH=arr(14, B, (4, 64), scale=MB + 128), nb=0) == -5


def test_top_logits():
    x, v = arr(1, B, (4, 104)), arr(2, B, (4, 8))

    def top(X=x, V=v, ids=IDS, lse=LSE):
        return sc.lib().scalify_scaled_top_logits(R(X), 1.0, R(V), ids, lse, None)

    for at in (MB + 4, 2 * MB + 4, IDS + 4, LSE + 4):
        assert top(V=arr(2, B, (4, 8), scale=at)) == ALIAS
    for at in (2 * MB + 4, IDS + 4, LSE + 4):
        assert top(X=arr(1, B, (4, 104), scale=at)) == ALIAS
