"""CPU tests: pins of the oracle of the fine-tuning operations, the generator's test vectors among them, and the
descriptions that the library refuses, which needs no GPU to say so."""
import ctypes as C

import numpy as np
import pytest

import paper_2002_05645_amd as P
from paper_2002_05645_amd import binding as B
from oracle import finetune_oracle as F


def test_generator_gives_the_published_vectors():
    # Philox-4x32 with ten and with seven rounds, counters and keys of all zeros and all ones (the test vectors of the publication's own code)
    def words(c, seed, rounds):
        return [int(x) for x in F.philox(c, c, c, c, seed, rounds)]
    ones = 0xFFFFFFFF
    assert words(0, 0, 10) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert words(ones, ones << 32 | ones, 10) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words(0, 0, 7) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    assert words(ones, ones << 32 | ones, 7) == [0x5207DDC2, 0x45165E59, 0x4D8EE751, 0x8C52F662]


def test_masks_drop_their_share_and_differ_by_site_seed_and_pair():
    z = F.drop_factors_attention(512, 3, 0.1, 77, 5)
    kept = (z > 0).mean()
    assert abs(kept - 230 / 256) < 5 * np.sqrt(0.1 * 0.9 / z.size)          # five standard deviations of a binomial share
    assert set(np.unique(z)) == {0.0, 256 / 230}
    for other in (F.drop_factors_attention(512, 4, 0.1, 77, 5), F.drop_factors_attention(512, 3, 0.1, 78, 5), F.drop_factors_attention(512, 3, 0.1, 77, 5 + (1 << 32))):
        same = ((z > 0) == (other > 0)).mean()
        assert abs(same - (kept ** 2 + (1 - kept) ** 2)) < 5 * np.sqrt(0.2 / z.size)
    y = F.drop_factors_rows(300, 333, 0.25, 1 << 40, 9)
    assert abs((y > 0).mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / y.size)


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients_against_differences(causal):
    rng = np.random.default_rng(0)
    n, d = 7, 5
    q, k, v, do = (rng.normal(size=(n, d)) for _ in range(4))
    Z = F.drop_factors_attention(n, 0, 0.3, 1, 2)
    loss = lambda q, k, v: (F.attention(q, k, v, 0.4, causal, Z)[0] * do).sum()  # noqa: E731
    P_ = F.attention(q, k, v, 0.4, causal, Z)[2]
    got = F.attention_bwd(q, k, v, 0.4, Z, P_, do)[:3]
    for which in range(3):
        num = np.zeros((n, d))
        for i in range(n):
            for c in range(d):
                args = [[x.copy() for x in (q, k, v)] for _ in range(2)]
                args[0][which][i, c] += 1e-5
                args[1][which][i, c] -= 1e-5
                num[i, c] = (loss(*args[0]) - loss(*args[1])) / 2e-5
        assert np.allclose(num, got[which], rtol=1e-6, atol=1e-8)


def test_logprob_gradients_against_differences():
    rng = np.random.default_rng(1)
    x, ids = rng.normal(size=(3, 9)) * 2, np.array([4, -1, 0])
    x[0, 2] = -np.inf
    g, h = rng.normal(size=3), rng.normal(size=3)
    loss = lambda x: (lambda r: (g * r[0]).sum() + (h * r[1]).sum())(F.token_logprobs(x, ids, 0))  # noqa: E731
    got = F.token_logprobs_bwd(x, ids, g, h)
    for i in range(3):
        for j in range(9):
            if np.isinf(x[i, j]):
                assert got[i, j] == 0
                continue
            a, b = x.copy(), x.copy()
            a[i, j] += 1e-5
            b[i, j] -= 1e-5
            assert abs((loss(a) - loss(b)) / 2e-5 - got[i, j]) < 1e-8
    # closed forms: equal logits have entropy log n; a lone finite logit has entropy 0 and probability 1
    lp, e, lse, order, top = F.token_logprobs(np.zeros((1, 8)), np.array([3]), 3)
    assert np.isclose(e[0], np.log(8)) and np.isclose(lp[0], -np.log(8)) and list(order[0]) == [0, 1, 2]
    x = np.full((1, 5), -np.inf)
    x[0, 4] = 3.0
    lp, e, lse, order, top = F.token_logprobs(x, np.array([4]), 2)
    assert lp[0] == 0 and e[0] == 0 and lse[0] == 3.0 and list(order[0]) == [4, 0] and top[0, 1] == -np.inf


def _description(**over):
    kw = dict(dtype="bf16", heads=4, kv_heads=2, head_dim=64, sequences=3, max_len=100)
    kw.update(over)
    return P.make_attention(**kw)


def test_attention_workspace_and_refused_descriptions():
    assert P.attention_work_bytes(_description()) >= 4 * 300 * 8
    assert P.attention_work_bytes(_description(dropout=0.1, causal=True, rows=301)) > 0
    for bad in (dict(dtype=3), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=12), dict(head_dim=0), dict(head_dim=136), dict(sequences=-1),
                dict(max_len=-1, rows=5), dict(max_len=262145, rows=1 << 20), dict(rows=299), dict(rows=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(dropout=1.0), dict(dropout=-0.1), dict(dropout=0.0019), dict(dropout=0.999), dict(dropout=float("nan")),
                dict(first=2), dict(length=2), dict(step=4), dict(sequences=1 << 20, max_len=1 << 17, rows=1 << 40)):
        assert P.attention_work_bytes(_description(**bad)) == 0, bad
    assert B.lib().l2l_op_attention_work_bytes(None) == 0
    for ok in (dict(dropout=0.00196), dict(dropout=0.998), dict(sequences=0), dict(max_len=0), dict(head_dim=8), dict(head_dim=128)):
        a = _description(**ok)
        assert P.attention_work_bytes(a) > 0 or a.rows == 0, ok


def test_other_workspaces_and_null_contexts():
    assert P.dropout_work_bytes(0, 5) == 0 and P.dropout_work_bytes(5, 0) == 0 and P.dropout_work_bytes(-1, 5) == 0
    assert P.dropout_work_bytes(1, 5) == 4 * 5
    assert P.dropout_work_bytes(32768, 1024) % (4 * 1024) == 0
    assert P.token_logprobs_work_bytes(0, 5, 1) == 0 and P.token_logprobs_work_bytes(5, 0, 1) == 0 and P.token_logprobs_work_bytes(5, 100, 33) == 0
    assert P.token_logprobs_work_bytes(5000, 30522, 5) == 0                  # as many rows as fill the chip: nothing to split
    L, a = B.lib(), _description()
    assert L.l2l_op_attention(None, C.byref(a), None, 0, None, 0, None, 0, None, 0, None, None) == P.L2L_E_ARG
    assert L.l2l_op_attention_bwd(None, C.byref(a), None, 0, None, 0, None, 0, None, 0, None, None, 0, None, 0, None, 0, None, 0, None) == P.L2L_E_ARG
    assert L.l2l_op_dropout(None, 1, 1, 8, None, 8, None, None, 0, None, 8, 0.1, 0, 0, None) == P.L2L_E_ARG
    assert L.l2l_op_dropout_bwd(None, 1, 1, 8, None, 8, None, 8, 0.1, 0, 0, None, None, 0, None) == P.L2L_E_ARG
    assert L.l2l_op_token_logprobs(None, 1, 1, 8, None, 8, None, None, None, None, 0, None, None, None) == P.L2L_E_ARG
    assert L.l2l_op_token_logprobs_bwd(None, 1, 1, 8, None, 8, None, None, None, None, None, None, 8) == P.L2L_E_ARG
