"""dblp_norm_rotate and its gradient refuse results of one side over what belongs to the other."""
import ctypes as C

import pytest

from paper_2605_01989_b200 import binding as dblp

EINVAL = -1
FAR = [(1 << 20) + (k << 24) for k in range(10)]       # addresses that are never read
SHAPE = dict(batch=2, tokens=16, q_heads=4, k_heads=4, head_dim=64, rotary_dim=64, dtype=1, weight_dtype=0, flags=0, eps=1e-6, positions=FAR[8],
             position_stride=16, freqs=FAR[8])


def heads(data):
    return C.byref(dblp.dblp_heads_t(data, 16 * 4 * 64, 4 * 64, 64))


@pytest.mark.parametrize("q,q_out,k,k_out,words", [
    (0, 2, 2, 3, "q_out lies over k"), (0, 1, 2, 0, "k_out lies over q"), (0, 1, 2, 1, "q_out lies over k_out"), (0, 2, 2, 0, "q_out lies over k"),
    (0, 0, 0, 3, "q_out lies over k")])
def test_norm_rotate_refuses_one_side_over_the_other(q, q_out, k, k_out, words):
    a = dblp.dblp_norm_rotate_t(**SHAPE)
    rc = dblp.lib().dblp_norm_rotate(C.byref(a), heads(FAR[q]), None, heads(FAR[q_out]), heads(FAR[k]), None, heads(FAR[k_out]), None)
    text = dblp.lib().dblp_last_error().decode()
    assert rc == EINVAL and words in text, (rc, text)


@pytest.mark.parametrize("dq,dk,dqw,dkw,words", [
    (2, 5, None, None, "dq lies over k"), (3, 5, None, None, "dq lies over dk_out"), (4, 0, None, None, "dk lies over q"), (4, 1, None, None, "dk lies over dq_out"),
    (4, 4, None, None, "dq lies over dk"), (4, 5, FAR[6], FAR[6], "dq_weight lies over dk_weight"), (4, 5, FAR[6], FAR[6] + 252, "dq_weight lies over dk_weight"),
    (4, 5, FAR[6] + 252, FAR[6], "dq_weight lies over dk_weight")])
def test_norm_rotate_grad_refuses_one_side_over_the_other(dq, dk, dqw, dkw, words):
    a = dblp.dblp_norm_rotate_t(**SHAPE)
    rc = dblp.lib().dblp_norm_rotate_grad(C.byref(a), heads(FAR[0]), None, heads(FAR[1]), heads(FAR[dq]), dqw, heads(FAR[2]), None, heads(FAR[3]),
                                          heads(FAR[dk]), dkw, FAR[7], 1 << 22, None)
    text = dblp.lib().dblp_last_error().decode()
    assert rc == EINVAL and words in text, (rc, text)
