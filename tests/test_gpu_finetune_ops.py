"""GPU tests of the single fine-tuning operations (attention over sequences of different lengths, dropout, token log
probabilities), through the C ABI, against the fp64 oracle.

Tolerances are sums of the roundings that a result goes through, entry by entry, from the oracle's own arrays: u = half a step
of the format for each value rounded to it (2^-8 bf16, 2^-11 fp16, 2^-24 fp32), and for fp32 sums and exponentials a multiple of 2^-24."""
import numpy as np
import pytest
import torch

import paper_2002_05645_amd as P
from oracle import finetune_oracle as F
from oracle import l2l_oracle as O
from gpu_util import to_host

pytestmark = pytest.mark.gpu

TDT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LOW = {"fp32": 2.0 ** -126, "bf16": 2.0 ** -126, "fp16": 2.0 ** -25}   # what a value below the format's normal range may lose
E24 = 2.0 ** -24
SEED, SITE = 0x1234_5678_9ABC_DEF1, (7 << 32) + 3


@pytest.fixture(scope="module")
def ctx():
    c = P.Context(P.make_config(64, 2, 128, 16, 2, 2, "bf16", 1e-5, 0))
    yield c
    c.close()


def dev_i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------- attention
class Problem:
    """Inputs of an attention call with every row that belongs to no sequence poisoned with NaN, and the outputs prefilled."""

    def __init__(self, dtype, heads, kv, d, lengths, causal=False, p=0.0, gaps=None, order=None, pad_cols=0, seed=0, amp=1.0, split_kv=False):
        self.dtype, self.heads, self.kv, self.d, self.lengths, self.causal, self.p = dtype, heads, kv, d, lengths, causal, p
        gaps = gaps or [0] * len(lengths)
        self.first, row = [], 0
        place = order or range(len(lengths))
        at = {}
        for b in place:
            row += gaps[b]
            at[b] = row
            row += lengths[b]
        self.first = [at[b] for b in range(len(lengths))]
        self.rows = row + 2
        g = torch.Generator().manual_seed(seed)
        t, Hq, Hk = TDT[dtype], heads * d, kv * d
        mine = torch.zeros(self.rows, dtype=torch.bool)
        for f, n in zip(self.first, lengths):
            mine[f:f + n] = True

        def matrix(cols, fill=float("nan")):
            x = torch.randn(self.rows, cols + pad_cols, generator=g) * amp
            x[~mine] = fill
            x[:, cols:] = fill
            return x.to(t).cuda()
        if split_kv:
            self.q, self.k, self.v = matrix(Hq), matrix(Hk), matrix(Hk)
        else:      # column groups of one projection
            self.qkv = matrix(Hq + 2 * Hk)
            self.q, self.k, self.v = self.qkv[:, :Hq], self.qkv[:, Hq:Hq + Hk], self.qkv[:, Hq + Hk:]
        self.do = matrix(Hq)
        out = lambda cols: torch.full((self.rows, cols + pad_cols), 7.0, dtype=t, device="cuda")  # noqa: E731
        self.o, self.dq, self.dk, self.dv = out(Hq), out(Hq), out(Hk), out(Hk)
        self.lse = torch.full((heads, self.rows), 7.0, device="cuda")
        self.mine = mine.numpy()
        self.plan = P.make_attention(dtype=dtype, heads=heads, kv_heads=kv, head_dim=d, sequences=len(lengths), max_len=max(lengths + [1]), rows=self.rows,
                                     first=dev_i32(self.first), length=dev_i32(lengths), causal=causal, dropout=p, seed=SEED, site=SITE)
        self.work = torch.full((P.attention_work_bytes(self.plan),), 255, dtype=torch.uint8, device="cuda")

    def forward(self, ctx):
        ctx.op_attention(self.plan, self.q, self.q.stride(0), self.k, self.k.stride(0), self.v, self.v.stride(0), self.o, self.o.stride(0), self.lse, self.work)

    def backward(self, ctx):
        ctx.op_attention_bwd(self.plan, self.q, self.q.stride(0), self.k, self.k.stride(0), self.v, self.v.stride(0), self.o, self.o.stride(0), self.lse,
                             self.do, self.do.stride(0), self.dq, self.dq.stride(0), self.dk, self.dk.stride(0), self.dv, self.dv.stride(0), self.work)

    def check(self, seqs=None, heads=None, scale=None):
        """every entry of o, lse, dq, dk, dv against the oracle, and that nothing else was written"""
        d, scale, u, low = self.d, self.d ** -0.5 if scale is None else scale, U[self.dtype], LOW[self.dtype]
        host = {x: to_host(getattr(self, x)) for x in ("q", "k", "v", "do", "o", "dq", "dk", "dv", "lse")}
        for x in ("o", "dq", "dk", "dv"):
            cols = d * (self.heads if x in ("o", "dq") else self.kv)
            assert (host[x][~self.mine] == 7).all() and (host[x][:, cols:] == 7).all(), x + ": wrote outside the sequences"
        assert (host["lse"][:, ~self.mine] == 7).all()
        G = self.heads // self.kv
        for b, n in enumerate(self.lengths):
            if n == 0 or (seqs is not None and b not in seqs):
                continue
            r = slice(self.first[b], self.first[b] + n)
            for hk in range(self.kv):
                ck = slice(hk * d, hk * d + d)
                k, v = host["k"][r, ck], host["v"][r, ck]
                dk_ref, dv_ref, dk_tol, dv_tol = 0, 0, 0, 0
                for h in range(hk * G, hk * G + G):
                    c = slice(h * d, h * d + d)
                    q, do = host["q"][r, c], host["do"][r, c]
                    Z = F.drop_factors_attention(n, b * self.heads + h, self.p, SEED, SITE)
                    o, lse, prob = F.attention(q, k, v, scale, self.causal, Z)
                    dq, dk, dv, dS = F.attention_bwd(q, k, v, scale, Z, prob, do)
                    used = prob * Z
                    # fp32 work: sums of d and n terms, exponents up to the largest |score| plus |lse|, a few single operations
                    mag = scale * (np.abs(q) @ np.abs(k).T)
                    f = ((n + d + 32) + 4 * (mag.max() + np.abs(lse).max())) * E24
                    absv, absdo, absk, absq = np.abs(v), np.abs(do), np.abs(k), np.abs(q)
                    uP = 0.0 if self.dtype == "fp32" else u      # P and dS as the matrix cores take them
                    o_in = (uP + f) * (used @ absv) + n * low * absv.max()     # before o itself is rounded
                    o_tol = o_in + u * (np.abs(o) + o_in) + low
                    err = np.abs(host["o"][r, c] - o)
                    assert (err <= o_tol).all(), ("o", b, h, n, (err / o_tol).max())
                    lse_tol = (d + n + 32 + 2 * mag.max()) * E24 + E24 * np.abs(lse)
                    assert (np.abs(host["lse"][h, r] - lse) <= lse_tol).all(), ("lse", b, h, n)
                    # D = rowsum(dO o) from the rounded o
                    dD = (absdo * o_tol).sum(-1) + f * (absdo * np.abs(o)).sum(-1)
                    dPabs = (absdo @ absv.T) * Z
                    dS_tol = uP * np.abs(dS) + prob * dD[:, None] + f * prob * (dPabs + (absdo * np.abs(o)).sum(-1)[:, None]) + f * np.abs(dS)
                    dS_tol = dS_tol * (1 + u) + low
                    dq_in = scale * (dS_tol @ absk) + f * scale * (np.abs(dS) @ absk)
                    dq_tol = dq_in + u * (np.abs(dq) + dq_in) + low
                    err = np.abs(host["dq"][r, c] - dq)
                    assert (err <= dq_tol).all(), ("dq", b, h, n, (err / dq_tol).max())
                    dk_ref, dv_ref = dk_ref + dk, dv_ref + dv
                    dk_tol = dk_tol + scale * (dS_tol.T @ absq) + G * f * scale * (np.abs(dS).T @ absq)
                    dv_tol = dv_tol + (uP + G * f) * (used.T @ absdo) + n * low * absdo.max()
                for name, ref, tol in (("dk", dk_ref, dk_tol), ("dv", dv_ref, dv_tol)):
                    tol = tol + u * (np.abs(ref) + tol) + low
                    err = np.abs(host[name][r, ck] - ref)
                    assert (err <= tol).all(), (name, b, hk, n, (err / tol).max())


EDGES = [1, 0, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,heads,kv,d", [("bf16", 2, 2, 64), ("fp16", 4, 2, 64), ("fp32", 2, 1, 64), ("bf16", 3, 1, 128), ("fp16", 2, 2, 96), ("bf16", 2, 1, 32),
                                              ("fp32", 2, 2, 128), ("bf16", 2, 2, 8), ("fp16", 1, 1, 40), ("fp32", 3, 3, 72), ("fp32", 1, 1, 24), ("bf16", 1, 1, 120)])
def test_attention_edges_of_the_tiles(ctx, dtype, heads, kv, d, causal):
    # lengths around every tile edge, packed out of order with gaps between them; probabilities dropped in the second pass
    gaps = [(3 * b) % 5 for b in range(len(EDGES))]
    order = [5, 2, 0, 1, 11, 3, 4, 10, 6, 9, 7, 8]
    for p in (0.0, 0.3):
        x = Problem(dtype, heads, kv, d, EDGES, causal, p, gaps, order, pad_cols=8, seed=d + heads)
        x.forward(ctx)
        x.backward(ctx)
        ctx.sync()
        x.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("fp16", 128), ("fp32", 96)])
def test_attention_longer_sequences_and_large_scores(ctx, dtype, d):
    # several hundred keys: the running maximum moves; scores of +-40, where a softmax row is a few entries
    x = Problem(dtype, 2, 1, d, [700, 513, 2], True, 0.1, seed=3, amp=2.5 if dtype != "fp32" else 2.0, split_kv=True)
    x.forward(ctx)
    x.backward(ctx)
    ctx.sync()
    x.check()


def test_attention_default_layout_and_one_long_sequence(ctx):
    # no arrays: sequences of max_len rows one after the other; 4099 tokens: many key tiles, a ragged end
    n, h, d = 4099, 1, 64
    x = Problem("bf16", h, h, d, [n], True, 0.0, seed=9)
    plan = P.make_attention(dtype="bf16", heads=h, head_dim=d, sequences=1, max_len=n, rows=x.rows, causal=True)
    x.plan = plan
    x.forward(ctx)
    x.backward(ctx)
    ctx.sync()
    x.check()
    y = Problem("bf16", h, h, d, [64] * 5, False, 0.0, seed=10)
    y.plan = P.make_attention(dtype="bf16", heads=h, head_dim=d, sequences=5, max_len=64, rows=y.rows)
    y.forward(ctx)
    y.backward(ctx)
    ctx.sync()
    y.check()


def test_attention_many_heads_share_one_key_head(ctx):
    for dtype in ("bf16", "fp32"):
        x = Problem(dtype, 16, 1, 64, [150, 70, 1], False, 0.1, seed=4)
        x.forward(ctx)
        x.backward(ctx)
        ctx.sync()
        x.check()


def test_attention_rows_far_behind_32_bit_offsets(ctx):
    # sequences whose first elements lie beyond 2^31 elements of every matrix
    rows, ld, d = 530000, 4160, 64
    big = torch.empty(rows, ld, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(rows, ld, dtype=torch.bfloat16, device="cuda")
    n, f = 130, rows - 131
    small = Problem("bf16", 1, 1, d, [n], False, 0.0, seed=5)
    big[f:f + n, :192] = small.qkv[:n, :192]
    big[f:f + n, 192:256] = small.do[:n]
    assert f * ld > 2 ** 31
    plan = P.make_attention(dtype="bf16", heads=1, head_dim=d, sequences=1, max_len=n, rows=rows, first=dev_i32([f]))
    lse, work = torch.empty(1, rows, device="cuda"), torch.empty(P.attention_work_bytes(plan), dtype=torch.uint8, device="cuda")
    q, k, v, do = (big[:, c:c + d] for c in (0, 64, 128, 192))
    o, dq, dk, dv = (out[:, c:c + d] for c in (0, 64, 128, 192))
    ctx.op_attention(plan, q, ld, k, ld, v, ld, o, ld, lse, work)
    ctx.op_attention_bwd(plan, q, ld, k, ld, v, ld, o, ld, lse, do, ld, dq, ld, dk, ld, dv, ld, work)
    ctx.sync()
    for name, x in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        getattr(small, name)[:n] = x[f:f + n]
    small.lse[:, :n] = lse[:, f:f + n]
    small.check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,heads,kv,d", [("bf16", 4, 1, 64), ("fp16", 3, 3, 96), ("bf16", 2, 2, 32), ("fp16", 4, 2, 128), ("bf16", 3, 1, 40), ("fp16", 1, 1, 8), ("fp32", 4, 1, 64), ("fp32", 2, 2, 128),
                                              ("fp32", 3, 1, 24)])
def test_attention_few_workgroups_share_the_long_axis(ctx, dtype, heads, kv, d, causal):
    # so few (sequence, head, block)s that the workgroups take parts of the keys, or of the queries, and a second kernel adds them up; splits that end
    # in the middle of a causal row, and short sequences whose splits are empty
    for p in (0.0, 0.3):
        x = Problem(dtype, heads, kv, d, [1100, 0, 1, 65, 130, 897], causal, p, gaps=[1, 0, 3, 0, 2, 1], pad_cols=8, seed=d, amp=1.5)
        assert x.work.numel() >= heads * x.rows * 8 + 2 * heads * x.rows * d * 4
        x.forward(ctx)
        x.backward(ctx)
        ctx.sync()
        x.check()


def test_attention_fp32_gradients_of_shared_heads_in_parts(ctx):
    # two waves on a tile pair, and parts that begin and end in the middle of a head's tiles
    for lengths in ([64, 40], [33, 64, 1, 0]):
        for causal in (False, True):
            x = Problem("fp32", 14, 2, 64, lengths, causal, 0.2, seed=14)
            assert x.work.numel() >= 14 * x.rows * 8 + 2 * 2 * 2 * x.rows * 64 * 4
            x.forward(ctx)
            x.backward(ctx)
            ctx.sync()
            x.check()


def test_attention_forward_without_workspace_is_not_split(ctx):
    x = Problem("bf16", 2, 2, 64, [1500], False, 0.2, seed=2)
    x.work, keep = None, x.work
    x.forward(ctx)
    x.work = keep
    x.backward(ctx)
    ctx.sync()
    x.check()


@pytest.mark.parametrize("dtype,heads,kv,d", [("bf16", 4, 2, 64), ("fp16", 6, 2, 32), ("bf16", 3, 1, 40)])
def test_attention_backward_in_one_kernel(ctx, dtype, heads, kv, d):
    # every sequence's keys fit one workgroup; lengths around the tile and wave edges, shared key heads, and a batch that leaves rows out
    for causal in (False, True):
        for p in (0.0, 0.3):
            x = Problem(dtype, heads, kv, d, [128, 127, 97, 96, 65, 64, 63, 33, 32, 31, 2, 1, 0, 100], causal, p, gaps=[0, 1] * 7, pad_cols=8, seed=heads)
            x.forward(ctx)
            x.backward(ctx)
            ctx.sync()
            x.check()


@pytest.mark.parametrize("heads,kv,d", [(2, 2, 64), (4, 2, 24), (3, 1, 96), (2, 1, 128), (4, 4, 40)])
def test_attention_short_fp32_sequences(ctx, heads, kv, d):
    # no sequence beyond 64: two waves on a row block's tiles, and query tiles of several heads in turn
    for causal in (False, True):
        for p in (0.0, 0.3):
            for lengths in ([64, 63, 33, 32, 31, 1, 0, 40], [20, 5], [64]):
                x = Problem("fp32", heads, kv, d, lengths, causal, p, gaps=[0, 1] * 4, pad_cols=8, seed=d)
                x.forward(ctx)
                x.backward(ctx)
                ctx.sync()
                x.check()


@pytest.mark.parametrize("dtype,d,longest", [("bf16", 64, 33), ("fp16", 32, 128), ("bf16", 96, 40), ("fp16", 128, 32), ("bf16", 64, 600)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_one_key_has_no_score_gradient(ctx, dtype, d, longest, causal):
    # a row that sees one key has the probability 1 whatever its score: dS = 0, although D = dO . O comes from a rounded O
    for p in (0.0, 0.4):
        x = Problem(dtype, 2, 1, d, [1, longest, 1, 20, 1], causal, p, seed=longest, amp=2.0)
        x.forward(ctx)
        x.backward(ctx)
        ctx.sync()
        x.check()
        for b, n in enumerate(x.lengths):
            if n > 1 and not causal:
                continue
            r = x.first[b]
            for h in range(2):
                c = slice(h * d, h * d + d)
                q, do, dq = (to_host(m[r, c]) for m in (x.q, x.do, x.dq))
                k, v = to_host(x.k[r, :d]), to_host(x.v[r, :d])
                # dP and D: sums of d terms and O's rounding; P = 1 within the fp32 work of one exponential; what is left of dS is their product
                f = (d + 64 + 8 * d ** -0.5 * (np.abs(q) @ np.abs(k))) * E24
                dP = np.abs(do) @ np.abs(v) / (1 - p)
                tol = d ** -0.5 * np.abs(k) * ((U[dtype] + f) * dP * f + 4 * E24 * (U[dtype] + f) * dP) * 2 + LOW[dtype]
                assert (np.abs(dq) <= tol).all(), (b, h, (np.abs(dq) / tol).max())


@pytest.mark.parametrize("heads,kv", [(9, 9), (16, 8), (18, 9)])
def test_attention_workgroups_by_xcd(ctx, heads, kv):
    # keys of one head that fill half an L2, and key heads that do not come in eights: every (head, block) is run once
    n, d = 8200, 128
    g = torch.Generator().manual_seed(heads)
    q, k, v = (torch.randn(n, h * d, generator=g).bfloat16().cuda() for h in (heads, kv, kv))
    o = torch.full((n, heads * d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((heads, n), 7.0, device="cuda")
    plan = P.make_attention(dtype="bf16", heads=heads, kv_heads=kv, head_dim=d, sequences=1, max_len=n, rows=n)
    ctx.op_attention(plan, q, heads * d, k, kv * d, v, kv * d, o, heads * d, lse)
    ctx.sync()
    rows = [0, 31, 127, 128, 4095, 8063, 8064, 8191, 8192, 8199]
    for h in range(heads):
        c, ck = slice(h * d, h * d + d), slice(h // (heads // kv) * d, h // (heads // kv) * d + d)
        Q, K, V = to_host(q[rows][:, c]), to_host(k[:, ck]), to_host(v[:, ck])
        S = (Q @ K.T) * d ** -0.5
        top = S.max(-1, keepdims=True)
        prob = np.exp(S - top)
        ref = (prob / prob.sum(-1, keepdims=True)) @ V
        ref_lse = top[:, 0] + np.log(prob.sum(-1))
        absv = (prob / prob.sum(-1, keepdims=True)) @ np.abs(V)
        # P rounded to the format, sums of n and d terms in fp32, the result rounded
        f = ((n + d + 32) + 8 * np.abs(S).max()) * E24
        assert (np.abs(to_host(o[rows][:, c]) - ref) <= (U["bf16"] + f) * absv * (1 + U["bf16"]) + U["bf16"] * np.abs(ref)).all(), h
        assert (np.abs(to_host(lse[h][rows]) - ref_lse) <= (d + n + 32 + 2 * np.abs(S).max()) * E24 + E24 * np.abs(ref_lse)).all(), h
    assert not (o == 7.0).all(-1).any()


def test_attention_same_call_gives_the_same_bits(ctx):
    x = Problem("bf16", 8, 2, 64, [300, 257, 64], True, 0.1, seed=6)
    x.forward(ctx)
    x.backward(ctx)
    first = [t.clone() for t in (x.o, x.lse, x.dq, x.dk, x.dv)]
    for _ in range(3):
        x.work.fill_(255)
        x.forward(ctx)
        x.backward(ctx)
        ctx.sync()
        assert all(torch.equal(a, b) for a, b in zip(first, (x.o, x.lse, x.dq, x.dk, x.dv)))


def test_attention_a_row_is_the_same_in_any_batch(ctx):
    # the mask goes by the sequence's number, everything else by the sequence alone: without dropout a sequence's results do not depend on its neighbours
    x = Problem("fp16", 4, 2, 96, [77, 200, 130], True, 0.0, seed=7)
    x.forward(ctx)
    one = P.make_attention(dtype="fp16", heads=4, kv_heads=2, head_dim=96, sequences=1, max_len=200, rows=x.rows, first=dev_i32([x.first[1]]), causal=True)
    o2 = torch.full_like(x.o, 7.0)
    ctx.op_attention(one, x.q, x.q.stride(0), x.k, x.k.stride(0), x.v, x.v.stride(0), o2, o2.stride(0))
    ctx.sync()
    r = slice(x.first[1], x.first[1] + 200)
    assert torch.equal(x.o[r], o2[r])


def test_attention_sequences_that_do_not_fit_are_skipped_and_reported(ctx):
    x = Problem("bf16", 2, 2, 64, [40, 50, 60, 70], False, 0.0, seed=8)
    good = x.first
    bad_first = [good[0], -1, x.rows - 10, good[3]]
    bad_len = [40, 50, 60, 71]
    x.plan = P.make_attention(dtype="bf16", heads=2, head_dim=64, sequences=4, max_len=70, rows=x.rows, first=dev_i32(bad_first), length=dev_i32(bad_len))
    x.forward(ctx)
    with pytest.raises(P.L2LError, match="sequence"):
        ctx.sync()
    x.backward(ctx)
    with pytest.raises(P.L2LError, match="sequence"):
        ctx.sync()
    ctx.sync()
    x.lengths = [40]
    x.mine[:] = False
    x.mine[good[0]:good[0] + 40] = True
    x.check()


def test_attention_refusals(ctx):
    x = Problem("bf16", 4, 2, 64, [32, 32], seed=1)
    ld = x.q.stride(0)

    def fwd(plan=x.plan, q=x.q, ldq=ld, k=x.k, ldk=ld, v=x.v, ldv=ld, o=x.o, ldo=256, lse=x.lse, work=x.work):
        ctx.op_attention(plan, q, ldq, k, ldk, v, ldv, o, ldo, lse, work)

    def bwd(lse=x.lse, dq=x.dq, dk=x.dk, dv=x.dv, lddq=256, lddk=128, work=x.work, do=x.do):
        ctx.op_attention_bwd(x.plan, x.q, ld, x.k, ld, x.v, ld, x.o, 256, lse, do, 256, dq, lddq, dk, lddk, dv, 128, work)
    fwd()
    bwd()
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=x.q.data_ptr() + 2), dict(ldq=ld + 4), dict(ldq=248), dict(ldk=120), dict(ldo=255), dict(ldo=0), dict(ldv=-ld),
               dict(o=x.q), dict(o=x.v), dict(lse=x.lse.data_ptr() + 2), dict(work=x.work.data_ptr() + 8), dict(ldq=1 << 24)):
        with pytest.raises(P.L2LError):
            fwd(**kw)
    for kw in (dict(lse=None), dict(work=None), dict(dq=None), dict(dk=x.dv), dict(dv=x.dq), dict(dq=x.o), dict(dk=x.k), dict(lddq=248), dict(lddk=132), dict(do=None)):
        with pytest.raises(P.L2LError):
            bwd(**kw)
    bad = P.make_attention(dtype="bf16", heads=4, kv_heads=2, head_dim=64, sequences=2, max_len=32, rows=x.rows, dropout=1.0)
    with pytest.raises(P.L2LError, match="dropout"):
        fwd(plan=bad)
    none = P.make_attention(dtype="bf16", heads=4, kv_heads=2, head_dim=64, sequences=0, max_len=32, rows=x.rows)
    x.o.fill_(7.0)
    fwd(plan=none, lse=None, work=None)
    ctx.sync()
    assert (x.o == 7).all()


# ------------------------------------------------------------------------------------- dropout
def _rows(rows, n, ld, t, g, offset=0):
    """[rows, n] view with row stride ld that starts `offset` elements into an allocation; everything around it is 7"""
    flat = torch.full((rows * ld + offset + 16,), 7.0, dtype=t, device="cuda")
    v = flat[offset:offset + rows * ld].view(rows, ld)[:, :n]
    v.copy_(torch.randn(rows, n, generator=g).to(t))
    return flat, v


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,n,pad,offset", [(1, 1, 0, 0), (5, 7, 0, 1), (33, 8, 8, 0), (200, 129, 3, 1), (130, 1024, 0, 0), (64, 1157, 0, 3), (1, 6144, 0, 0), (4097, 24, 0, 0), (700, 520, 0, 0)])
def test_dropout_rows_of_any_alignment(ctx, dtype, rows, n, pad, offset):
    g = torch.Generator().manual_seed(rows + n)
    t, u, dt, ld = TDT[dtype], U[dtype], P.DTYPES[dtype], n + pad
    (_, x), (_, res), (yflat, y), (_, dy), (dxflat, dx) = (_rows(rows, n, ld, t, g, offset) for _ in range(5))
    bias = torch.randn(n, generator=g).to(t).cuda()
    work = torch.full((P.dropout_work_bytes(rows, n),), 255, dtype=torch.uint8, device="cuda")
    for p, b, r in ((0.1, bias, res), (0.5, None, None), (0.9, bias, None), (0.0, None, res)):
        yflat[:] = 7.0
        dxflat[:] = 7.0
        ctx.op_dropout(dt, rows, n, x, ld, y, ld, p, SEED, SITE, bias=b, resid=r, ldr=ld)
        dbias = torch.full((n,), 3.0, device="cuda")
        ctx.op_dropout_bwd(dt, rows, n, dy, ld, dx, ld, p, SEED, SITE, dbias=dbias, work=work)
        ctx.sync()
        Z = F.drop_factors_rows(rows, n, p, SEED, SITE)
        xin = to_host(x) + (to_host(b) if b is not None else 0.0)
        rin = to_host(r) if r is not None else 0.0
        ref = xin * Z + rin
        # bias, factor and residual each round to fp32 once, the result once to the format
        tol = u * np.abs(ref) + 4 * E24 * (np.abs(xin) * Z + np.abs(rin)) + LOW[dtype]
        assert (np.abs(to_host(y) - ref) <= tol).all(), (p, "y")
        if r is None:
            assert ((to_host(y) != 0) == ((Z > 0) & (xin != 0))).all(), "the mask is the generator's"
        gref = to_host(dy) * Z
        assert (np.abs(to_host(dx) - gref) <= (u + 2 * E24) * np.abs(gref) + LOW[dtype]).all(), (p, "dx")
        sref, sabs = gref.sum(0), np.abs(gref).sum(0)
        assert (np.abs(to_host(dbias) - sref) <= (rows + 2) * E24 * sabs).all(), (p, "dbias")
        old = dbias.clone()
        ctx.op_dropout_bwd(dt, rows, n, dy, ld, dx, ld, p, SEED, SITE, dbias=dbias, work=work, accumulate=True)
        ctx.sync()
        assert torch.equal(dbias, old + old)
        # outside the rows: nothing
        for flat in (yflat, dxflat):
            out = flat.clone()
            out[offset:offset + rows * ld].view(rows, ld)[:, :n] = 7.0
            assert (out == 7).all()


def test_dropout_in_place_strided_and_refused(ctx):
    g = torch.Generator().manual_seed(2)
    x = torch.randn(50, 40, generator=g).cuda()
    y = torch.empty(50, 40, device="cuda")
    ctx.op_dropout(P.L2L_F32, 50, 40, x, 40, y, 40, 0.25, 5, 6, resid=x, ldr=40)
    z = x.clone()
    ctx.op_dropout(P.L2L_F32, 50, 40, z, 40, z, 40, 0.25, 5, 6, resid=z, ldr=40)
    wide = torch.full((50, 64), 7.0, device="cuda")
    ctx.op_dropout(P.L2L_F32, 50, 40, x, 40, wide, 64, 0.25, 5, 6, resid=x, ldr=40)
    ctx.sync()
    assert torch.equal(y, z) and torch.equal(wide[:, :40], y) and (wide[:, 40:] == 7).all()
    work = torch.empty(P.dropout_work_bytes(50, 40), dtype=torch.uint8, device="cuda")
    sums = torch.full((40,), 2.0, device="cuda")
    for call in (lambda: ctx.op_dropout(7, 50, 40, x, 40, y, 40, 0.25, 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, -1, 40, x, 40, y, 40, 0.25, 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, 50, 40, None, 40, y, 40, 0.25, 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, 50, 40, x, 39, y, 40, 0.25, 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, 50, 40, x.data_ptr() + 2, 40, y, 40, 0.25, 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, 50, 40, x, 40, y, 40, 1.0, 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, 50, 40, x, 40, y, 40, 1e-6, 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, 50, 40, x, 40, y, 40, float("nan"), 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, 50, 40, x, 40, y, 40, 0.25, 5, 6, resid=x, ldr=39),
                 lambda: ctx.op_dropout(P.L2L_F32, 25, 40, x, 40, x, 80, 0.25, 5, 6),
                 lambda: ctx.op_dropout(P.L2L_F32, 50, 40, x, 40, y, 40, 0.25, 5, 6, step=4),
                 lambda: ctx.op_dropout_bwd(P.L2L_F32, 50, 40, x, 40, y, 40, 0.25, 5, 6, dbias=sums),
                 lambda: ctx.op_dropout_bwd(P.L2L_F32, 50, 40, x, 40, y, 40, 0.25, 5, 6, dbias=sums, work=work.data_ptr() + 4)):
        with pytest.raises(P.L2LError):
            call()
    ctx.op_dropout(P.L2L_F32, 0, 40, None, 40, None, 40, 0.25, 5, 6)
    ctx.op_dropout_bwd(P.L2L_F32, 0, 40, None, 40, None, 40, 0.25, 5, 6, dbias=sums, work=work, accumulate=True)
    ctx.sync()
    assert (sums == 2).all()
    ctx.op_dropout_bwd(P.L2L_F32, 0, 40, None, 40, None, 40, 0.25, 5, 6, dbias=sums, work=work)
    ctx.sync()
    assert (sums == 0).all()


# ------------------------------------------------------------------------------------- token log probabilities
def _logprobs(ctx, dtype, x, ids, top, ld=None, work=True, g=None, h=None, in_place=False):
    rows, vocab = x.shape
    t, dt = TDT[dtype], P.DTYPES[dtype]
    ld = ld or vocab
    buf = torch.full((rows, ld), float("nan"), dtype=t, device="cuda")
    buf[:, :vocab] = torch.as_tensor(x).to(t)
    idd = dev_i32(ids) if ids is not None else None
    logp = torch.full((rows,), 9.0, device="cuda") if ids is not None else None
    entropy, lse = torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
    top_ids = torch.full((rows, top), -5, dtype=torch.int32, device="cuda") if top else None
    top_logp = torch.full((rows, top), 9.0, device="cuda") if top else None
    nb = P.token_logprobs_work_bytes(rows, vocab, top) if work else 0
    wk = torch.full((nb,), 255, dtype=torch.uint8, device="cuda") if nb else None
    ctx.op_token_logprobs(dt, rows, vocab, buf, ld, idd, logp, entropy, lse, top, top_ids, top_logp, wk)
    out = dict(x=to_host(buf[:, :vocab]), logp=logp, entropy=entropy, lse=lse, top_ids=top_ids, top_logp=top_logp)
    if g is not None:
        dx = buf if in_place else torch.full((rows, ld), 7.0, dtype=t, device="cuda")
        ctx.op_token_logprobs_bwd(dt, rows, vocab, buf, ld, idd, lse, entropy, g, h, dx, ld)
        out["dx"] = to_host(dx[:, :vocab])
        if not in_place:
            assert (dx[:, vocab:] == 7).all()
    torch.cuda.synchronize()
    return out


def _check_logprobs(r, ids, top, dtype, g=None, h=None):
    x = r["x"]
    n = x.shape[1]
    ids = np.asarray(ids)
    logp, entropy, lse, order, top_logp = F.token_logprobs(x, ids, top)
    fin = np.isfinite(x)
    span = np.array([np.ptp(row[f]) if f.any() else 0.0 for row, f in zip(x, fin)])
    most = np.array([np.abs(row[f]).max() if f.any() else 0.0 for row, f in zip(x, fin)])
    # sums of at most 64 terms a thread and a dozen joins, exponentials of up to `span` (relative error: span roundings of the argument), logarithms
    f = (96 + 4 * span) * E24
    same = lambda a, b, tol: ((np.abs(a - b) <= tol) | (a == b)).all()  # noqa: E731
    with np.errstate(invalid="ignore"):
        assert same(to_host(r["lse"]), lse, f + 4 * E24 * most)
        assert same(to_host(r["logp"]), logp, f + 4 * E24 * (span + 32))
        assert same(to_host(r["entropy"]), entropy, 2 * f * (1 + span))
        if top:
            assert np.array_equal(r["top_ids"].cpu().numpy(), order)
            assert same(to_host(r["top_logp"]), top_logp, (f + 4 * E24 * (span + 32))[:, None])
    if g is not None:
        gh, hh = to_host(g), to_host(h)
        ref = F.token_logprobs_bwd(x, ids, gh, hh)
        with np.errstate(invalid="ignore"):
            p = np.exp(np.where(fin, x - lse[:, None], -np.inf))
        p[~np.isfinite(p)] = 0
        size = np.abs(gh)[:, None] * (ids >= 0)[:, None] + np.abs(hh)[:, None] * (span + 2 * np.log(n) + 2)[:, None]
        tol = U[dtype] * np.abs(ref) + (8 * f + 8 * E24 * most)[:, None] * p * size + 2 * E24 * np.abs(ref) + LOW[dtype]
        err = np.abs(r["dx"] - ref)
        assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,vocab,top", [(3, 1, 1), (5, 2, 2), (4, 63, 5), (300, 100, 0), (7, 511, 32), (2, 2047, 3), (5, 4099, 10), (3, 8200, 32), (2, 30522, 5), (1, 40001, 7), (2, 128257, 20), (600, 1000, 4)])
def test_logprobs_and_gradients(ctx, dtype, rows, vocab, top):
    rng = np.random.default_rng(vocab + rows)
    x = (rng.normal(size=(rows, vocab)) * 3).astype(np.float32)
    ids = rng.integers(0, vocab, rows)
    ids[rows // 2] = -1 if rows > 1 else ids[0]
    g, h = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    for ld, work, in_place in ((vocab, True, False), (vocab + 5, False, True)):
        r = _logprobs(ctx, dtype, x, ids, top, ld, work, g, h, in_place)
        ctx.sync()
        _check_logprobs(r, ids, top, dtype, g, h)


@pytest.mark.parametrize("dtype,vocab,rows", [("fp32", 5000, 3), ("bf16", 30522, 2), ("fp16", 70000, 400)])
def test_logprobs_equal_and_masked_logits(ctx, dtype, vocab, rows):
    # whole rows of equal logits, of two values, of -inf but one, of -inf alone, of a mask's lowest finite value
    x = np.zeros((rows, vocab), np.float32)
    x[0] = -0.0
    x[0, 1::2] = 0.0                     # zeros of either sign are equal
    x[1] = 2.0
    x[1, vocab // 2:] = 3.0
    ids = np.zeros(rows, int)
    ids[0] = vocab - 1
    if rows > 2:
        x[2] = -np.inf
        x[2, vocab - 3] = 1.5
        ids[2] = vocab - 3
    if rows > 3:
        x[3] = -np.inf                   # nothing is possible
        x[4] = np.finfo(np.float16).min
        x[4, 7] = 0.0
        x[5, 100:] = -np.inf
        ids[6] = -1
    g, h = torch.ones(rows, device="cuda"), torch.full((rows,), 0.5, device="cuda")
    for work in (True, False):
        r = _logprobs(ctx, dtype, x, ids, 9, work=work, g=g, h=h)
        ctx.sync()
        _check_logprobs(r, ids, 9, dtype, g, h)
        if rows > 3:
            assert to_host(r["lse"])[3] == -np.inf and to_host(r["entropy"])[3] == 0 and to_host(r["logp"])[3] == -np.inf and (r["dx"][3] == 0).all()


def test_logprobs_nan_and_infinity_stay_in_their_rows(ctx):
    rng = np.random.default_rng(3)
    x = rng.normal(size=(4, 9000)).astype(np.float32)
    x[1, 4000] = np.nan
    x[2, 17] = np.inf
    ids = np.array([1, 2, 3, 4])
    r = _logprobs(ctx, "fp32", x, ids, 6)
    ctx.sync()
    for name in ("logp", "entropy", "lse"):
        got = to_host(r[name])
        assert np.isnan(got[1]) and (np.isnan(got[2]) or got[2] == np.inf) and np.isfinite(got[[0, 3]]).all()
    top = r["top_ids"].cpu().numpy()
    assert ((top >= 0) & (top < 9000)).all() and top[2, 0] == 17
    good = [0, 3]
    ref = F.token_logprobs(x[good].astype(np.float64), ids[good], 6)
    assert np.array_equal(top[good], ref[3])


def test_logprobs_without_ids_and_ids_outside_the_vocabulary(ctx):
    x = np.random.default_rng(4).normal(size=(3, 500)).astype(np.float32)
    r = _logprobs(ctx, "fp32", x, None, 4)
    ctx.sync()
    assert np.array_equal(r["top_ids"].cpu().numpy(), F.token_logprobs(x.astype(np.float64), np.zeros(3, int), 4)[3])
    _logprobs(ctx, "fp32", x, [1, 500, 2], 0)
    with pytest.raises(P.L2LError, match="token id"):
        ctx.sync()
    ctx.sync()


def test_logprobs_refusals(ctx):
    x, f, i = torch.zeros(4, 100, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")

    def fwd(dt=P.L2L_F32, rows=4, vocab=100, logits=x, ld=100, ids=i, logp=f, entropy=f, lse=f, top=2, top_ids=i, top_logp=f, work=None):
        ctx.op_token_logprobs(dt, rows, vocab, logits, ld, ids, logp, entropy, lse, top, top_ids, top_logp, work)

    def bwd(ids=i, lse=f, entropy=f, dlogp=f, dentropy=f, dlogits=x, ldd=100):
        ctx.op_token_logprobs_bwd(P.L2L_F32, 4, 100, x, 100, ids, lse, entropy, dlogp, dentropy, dlogits, ldd)
    fwd(top_logp=f[32:], lse=f[16:])
    bwd()
    for kw in (dict(dt=5), dict(rows=-1), dict(vocab=0), dict(vocab=101), dict(logits=None), dict(logits=x.data_ptr() + 1), dict(ids=None), dict(logp=None), dict(entropy=None), dict(lse=None),
               dict(top=33), dict(top=-1), dict(top_ids=None), dict(top_logp=None), dict(work=f.data_ptr() + 4), dict(vocab=1, top=2), dict(rows=1 << 30, vocab=1 << 20, ld=1 << 20)):
        with pytest.raises(P.L2LError):
            fwd(**kw)
    for kw in (dict(ids=None), dict(lse=None), dict(entropy=None), dict(dlogits=None), dict(ldd=99), dict(ldd=104), dict(dlogits=x.data_ptr() + 2)):
        with pytest.raises(P.L2LError):
            bwd(**kw)
    fwd(rows=0, logits=None)
    ctx.sync()


# ------------------------------------------------------------------------------------- together
def _captured(stream, body):
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        body()
    return graph


def test_captured_calls_replay_and_take_a_new_mask_with_the_step():
    stream = torch.cuda.Stream()
    c = P.Context(P.make_config(64, 2, 128, 16, 2, 2, "bf16", 1e-5, 0), stream.cuda_stream, stream.cuda_stream)
    try:
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        x = Problem("bf16", 4, 2, 64, [100, 33, 1], True, 0.2, seed=11)
        x.plan = P.make_attention(dtype="bf16", heads=4, kv_heads=2, head_dim=64, sequences=3, max_len=100, rows=x.rows, first=dev_i32(x.first), length=dev_i32(x.lengths), causal=True,
                                  dropout=0.2, seed=SEED, site=SITE, step=step)
        g = torch.Generator().manual_seed(1)
        y = torch.randn(70, 256, generator=g).to(torch.bfloat16).cuda()
        z, dz = torch.empty_like(y), torch.empty_like(y)
        dbias, wk = torch.empty(256, device="cuda"), torch.empty(P.dropout_work_bytes(70, 256), dtype=torch.uint8, device="cuda")
        logits = torch.randn(2, 9000, generator=g).cuda()
        ids = dev_i32([5, 8999])
        outs = [torch.empty(2, device="cuda") for _ in range(3)]
        tid, tlp = torch.empty(2, 4, dtype=torch.int32, device="cuda"), torch.empty(2, 4, device="cuda")
        lwk = torch.empty(P.token_logprobs_work_bytes(2, 9000, 4), dtype=torch.uint8, device="cuda")
        dl = torch.empty_like(logits)

        def body():
            x.forward(c)
            x.backward(c)
            c.op_dropout(P.L2L_BF16, 70, 256, y, 256, z, 256, 0.2, SEED, SITE, step=step)
            c.op_dropout_bwd(P.L2L_BF16, 70, 256, y, 256, dz, 256, 0.2, SEED, SITE, dbias=dbias, work=wk, step=step)
            c.op_token_logprobs(P.L2L_F32, 2, 9000, logits, 9000, ids, *outs, 4, tid, tlp, lwk)
            c.op_token_logprobs_bwd(P.L2L_F32, 2, 9000, logits, 9000, ids, outs[2], outs[1], outs[0], outs[1], dl, 9000)
        results = lambda: [t.clone() for t in (x.o, x.lse, x.dq, x.dk, x.dv, z, dz, dbias, *outs, tid, tlp, dl)]  # noqa: E731
        eager = []
        for s in range(3):
            step.fill_(s)
            torch.cuda.synchronize()
            body()
            torch.cuda.synchronize()
            eager.append(results())
        assert not torch.equal(eager[0][5], eager[1][5]) and not torch.equal(eager[0][0], eager[1][0])
        graph = _captured(stream, body)
        for s in (2, 0, 1, 0, 2):
            step.fill_(s)
            for t in (x.o, x.dq, x.dk, x.dv, z, dz, dbias, dl):
                t[:] = 7.0
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()
            torch.cuda.synchronize()
            torch.randn(1000, device="cuda").sum().item()      # the program's own work between replays
            assert all(torch.equal(a, b) for i, (a, b) in enumerate(zip(results(), eager[s])) if i not in (0, 2, 3, 4))
            for i in (0, 2, 3, 4):      # (rows of no sequence were refilled above)
                a, b = results()[i], eager[s][i]
                assert torch.equal(a[torch.from_numpy(x.mine)], b[torch.from_numpy(x.mine)])
    finally:
        c.close()


def test_captured_calls_in_parts_share_one_workspace():
    # two captured graphs (a training and an evaluation pass) over sequences long enough for parts, one workspace, replayed in turn
    stream = torch.cuda.Stream()
    c = P.Context(P.make_config(64, 2, 128, 16, 2, 2, "bf16", 1e-5, 0), stream.cuda_stream, stream.cuda_stream)
    try:
        for dtype in ("bf16", "fp32"):
            x = Problem(dtype, 4, 1, 64, [900, 70], True, 0.2, seed=31)
            calm = P.make_attention(dtype=dtype, heads=4, kv_heads=1, head_dim=64, sequences=2, max_len=900, rows=x.rows, first=dev_i32(x.first), length=dev_i32(x.lengths))
            assert P.attention_work_bytes(calm) == P.attention_work_bytes(x.plan) > 4 * x.rows * 8
            train = x.plan

            def body():
                x.forward(c)
                x.backward(c)
            graphs, eager = [], []
            for plan, what in ((train, body), (calm, lambda: x.forward(c))):
                x.plan = plan
                torch.cuda.synchronize()
                what()
                torch.cuda.synchronize()
                eager.append([t.clone() for t in (x.o, x.lse, x.dq, x.dk, x.dv)])
                graphs.append(_captured(stream, what))
            for which in (0, 1, 0, 0, 1, 0):
                for t in (x.o, x.lse) if which else (x.o, x.lse, x.dq, x.dk, x.dv):
                    t.fill_(7.0)
                x.work.fill_(255)
                torch.cuda.synchronize()
                with torch.cuda.stream(stream):
                    graphs[which].replay()
                torch.cuda.synchronize()
                torch.randn(1000, device="cuda").sum().item()
                assert all(torch.equal(a, b) for a, b in zip((x.o, x.lse, x.dq, x.dk, x.dv)[:2 if which else 5], eager[which]))
            x.plan = train
            with torch.cuda.stream(stream):
                graphs[0].replay()
            torch.cuda.synchronize()
            x.check()
    finally:
        c.close()


def test_two_contexts_on_two_streams_at_once():
    streams = [torch.cuda.Stream() for _ in range(2)]
    cs = [P.Context(P.make_config(64, 2, 128, 16, 2, 2, "bf16", 1e-5, 0), s.cuda_stream, s.cuda_stream) for s in streams]
    try:
        xs = [Problem("bf16", 4, 2, 64, [300, 200], True, 0.1, seed=20 + i) for i in range(2)]
        torch.cuda.synchronize()
        for _ in range(3):
            for c, x in zip(cs, xs):
                x.forward(c)
                x.backward(c)
        for c, x in zip(cs, xs):
            c.sync()
            x.check()
    finally:
        for c in cs:
            c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_a_fine_tuning_layer_out_of_single_operations(ctx, dtype):
    """QKV projection, attention with dropped probabilities over sequences of different lengths, output projection, dropout with bias
    and residual, then logits, log probabilities and entropies, and every gradient back to the input: against the same chain in fp64."""
    H, A, V, lengths, p = 128, 2, 200, [64, 17, 1, 40], 0.1
    d, T = H // A, sum(lengths)
    first = [sum(lengths[:b]) for b in range(len(lengths))]
    rng = np.random.default_rng(12)
    t, dt = TDT[dtype], P.DTYPES[dtype]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(t).cuda()  # noqa: E731
    X, Wqkv, Wo, bo, E = dev(rng.normal(size=(T, H))), dev(rng.normal(size=(H, 3 * H)) / H ** 0.5), dev(rng.normal(size=(H, H)) / H ** 0.5), dev(rng.normal(size=H)), dev(rng.normal(size=(V, H)) * 0.2)
    ids = rng.integers(0, V, T)
    ids[3] = -1
    gl, ge = rng.normal(size=T).astype(np.float32) / T, rng.normal(size=T).astype(np.float32) / T
    new = lambda *s, dtype=t: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    qkv, o, out, y, z = new(T, 3 * H), new(T, H), new(T, H), new(T, H), new(T, V)
    plan = P.make_attention(dtype=dtype, heads=A, head_dim=d, sequences=len(lengths), max_len=max(lengths), rows=T, first=dev_i32(first), length=dev_i32(lengths), dropout=p, seed=SEED, site=1)
    lse, work = new(A, T, dtype=torch.float32), new(P.attention_work_bytes(plan), dtype=torch.uint8)
    f32 = dtype == "fp32"
    gemm = lambda a_kc, b_kc, M, N, K, a, lda, b, ldb, c, ldc: ctx.op_gemm(dt, f32, a_kc, b_kc, M, N, K, a, lda, b, ldb, c, ldc)  # noqa: E731
    gemm(1, 0, T, 3 * H, H, X, H, Wqkv, 3 * H, qkv, 3 * H)
    q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
    ctx.op_attention(plan, q, 3 * H, k, 3 * H, v, 3 * H, o, H, lse, work)
    gemm(1, 0, T, H, H, o, H, Wo, H, out, H)
    ctx.op_dropout(dt, T, H, out, H, y, H, p, SEED, 2, bias=bo, resid=X, ldr=H)
    gemm(1, 1, T, V, H, y, H, E, H, z, V)
    logp, ent, ls = (new(T, dtype=torch.float32) for _ in range(3))
    idd = dev_i32(ids)
    tid, tlp = new(T, 3, dtype=torch.int32), new(T, 3, dtype=torch.float32)
    ctx.op_token_logprobs(dt, T, V, z, V, idd, logp, ent, ls, 3, tid, tlp)
    dz, dy, dout, do, dqkv, dX = new(T, V), new(T, H), new(T, H), new(T, H), new(T, 3 * H), new(T, H)
    ctx.op_token_logprobs_bwd(dt, T, V, z, V, idd, ls, ent, torch.from_numpy(gl).cuda(), torch.from_numpy(ge).cuda(), dz, V)
    gemm(1, 0, T, H, V, dz, V, E, H, dy, H)
    dbo, wk = new(H, dtype=torch.float32), new(P.dropout_work_bytes(T, H), dtype=torch.uint8)
    ctx.op_dropout_bwd(dt, T, H, dy, H, dout, H, p, SEED, 2, dbias=dbo, work=wk)
    gemm(1, 1, T, H, H, dout, H, Wo, H, do, H)
    ctx.op_attention_bwd(plan, q, 3 * H, k, 3 * H, v, 3 * H, o, H, lse, do, H, dqkv[:, :H], 3 * H, dqkv[:, H:2 * H], 3 * H, dqkv[:, 2 * H:], 3 * H, work)
    ctx.op_gemm(dt, f32, 1, 1, T, H, 3 * H, dqkv, 3 * H, Wqkv, 3 * H, dX, H, resid=dy)
    ctx.sync()
    # the chain in fp64
    X_, Wq, Wo_, bo_, E_ = (to_host(a) for a in (X, Wqkv, Wo, bo, E))
    qkv_ = X_ @ Wq
    o_ = np.zeros((T, H))
    kept = []
    for b, (f, n) in enumerate(zip(first, lengths)):
        for h in range(A):
            r, c = slice(f, f + n), slice(h * d, h * d + d)
            qq, kk, vv = (qkv_[r, i * H + h * d:i * H + h * d + d] for i in range(3))
            Z = F.drop_factors_attention(n, b * A + h, p, SEED, 1)
            o_[r, c], _, prob = F.attention(qq, kk, vv, d ** -0.5, False, Z)
            kept.append((r, c, h, qq, kk, vv, Z, prob))
    Zr = F.drop_factors_rows(T, H, p, SEED, 2)
    y_ = (o_ @ Wo_ + bo_) * Zr + X_
    z_ = y_ @ E_.T
    logp_, ent_, _, _, _ = F.token_logprobs(z_, ids, 3)
    dz_ = F.token_logprobs_bwd(z_, ids, gl.astype(np.float64), ge.astype(np.float64))
    dy_ = dz_ @ E_
    dout_ = dy_ * Zr
    do_ = dout_ @ Wo_.T
    dqkv_ = np.zeros((T, 3 * H))
    for r, c, h, qq, kk, vv, Z, prob in kept:
        for i, gr in enumerate(F.attention_bwd(qq, kk, vv, d ** -0.5, Z, prob, do_[r, c])[:3]):
            dqkv_[r, i * H + h * d:i * H + h * d + d] = gr
    dX_ = dqkv_ @ Wq.T + dy_
    # up to a dozen roundings to the format stand between input and result; errors of independent roundings add up like their
    # squares, the products' factors are of size one: a dozen half steps bound the relative 2-norm with room to spare (fp32: sums as well)
    tol = 12 * U[dtype] if dtype != "fp32" else 2e-6
    for name, got, ref in (("logp", logp, logp_), ("entropy", ent, ent_), ("dlogits", dz, dz_), ("dbias", dbo, dout_.sum(0)), ("dqkv", dqkv, dqkv_), ("dX", dX, dX_)):
        assert O.rel_l2(to_host(got), ref) < tol, (name, O.rel_l2(to_host(got), ref))


def test_sizes_that_one_launch_does_not_hold_are_refused(ctx):
    x = torch.zeros(64, device="cuda")
    i = torch.zeros(64, dtype=torch.int32, device="cuda")
    with pytest.raises(P.L2LError, match="2\\^30"):
        ctx.op_dropout(P.DTYPES["fp32"], 2 ** 30 + 1, 8, x, 8, x, 8, 0.1, 1, 1)
    with pytest.raises(P.L2LError, match="2\\^30"):
        ctx.op_dropout(P.DTYPES["bf16"], 1, 2 ** 31 - 9, x, 2 ** 31, x, 2 ** 31, 0.1, 1, 1)
    with pytest.raises(P.L2LError, match="2\\^25"):
        ctx.op_dropout_bwd(P.DTYPES["fp32"], 1, 2 ** 25 + 1, x, 2 ** 26, x, 2 ** 26, 0.1, 1, 1, dbias=x, work=x)
    assert P.dropout_work_bytes(1, 2 ** 25 + 1) == 0 and P.dropout_work_bytes(2 ** 30 + 1, 8) == 0
    for rows, vocab in ((2 ** 22 + 1, 100), (2 ** 20, 2 ** 16)):
        with pytest.raises(P.L2LError, match="too many rows"):
            ctx.op_token_logprobs(P.DTYPES["bf16"], rows, vocab, x, vocab, i, x, x, x)
        with pytest.raises(P.L2LError, match="too many rows"):
            ctx.op_token_logprobs_bwd(P.DTYPES["bf16"], rows, vocab, x, vocab, i, x, x, x, None, x, vocab)
    for scale in (1e-30, 1e30, float("inf"), float("nan"), -1.0, 0.0):
        plan = P.make_attention(dtype="bf16", heads=1, head_dim=8, sequences=1, max_len=4, scale=scale)
        assert P.attention_work_bytes(plan) == 0
    plan = P.make_attention(dtype="bf16", heads=64, head_dim=8, sequences=2 ** 18, max_len=1, rows=2 ** 18)
    assert P.attention_work_bytes(plan) == 0
    ctx.sync()


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** -12, 0.7])
def test_attention_of_any_scale(ctx, scale):
    for dtype in ("bf16", "fp32"):
        x = Problem(dtype, 2, 1, 64, [200, 33, 2], True, 0.0, seed=3)
        x.plan = P.make_attention(dtype=dtype, heads=2, kv_heads=1, head_dim=64, sequences=3, max_len=200, rows=x.rows, first=dev_i32(x.first),
                                  length=dev_i32(x.lengths), causal=True, scale=scale)
        x.forward(ctx)
        x.backward(ctx)
        ctx.sync()
        x.check(scale=scale)
