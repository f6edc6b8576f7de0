"""GPU tests of the single fine-tuning operations at the ends of their numbers: masked and far-away logits, NaN, scores of any size, small
gradients, and what l2l_sync reports.

Expected values are computed in fp64 relative to each row's maximum, where a fill of the type's lowest value leaves nothing to cancel."""
import numpy as np
import pytest
import torch

import paper_2002_05645_amd as P
from oracle import finetune_oracle as F
from gpu_util import to_host
from test_gpu_finetune_ops import E24, LOW, SEED, SITE, TDT, U, Problem, _logprobs, ctx, dev_i32  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------- token log probabilities
def _row_reference(x, ids, top):
    """logp, entropy, lse, top ids, their log probabilities, log p of every token; x: rows of fp64 without NaN or +inf"""
    with np.errstate(invalid="ignore", divide="ignore"):
        m = x.max(-1, keepdims=True)
        d = np.where(np.isneginf(x), -np.inf, x - m)
        e = np.exp(d)
        s = e.sum(-1, keepdims=True)
        lp = d - np.log(s)
        entropy = np.log(s) - np.where(e > 0, e * np.where(e > 0, d, 0.0), 0.0).sum(-1, keepdims=True) / s
        lse = m + np.log(s)
    order = np.stack([np.lexsort((np.arange(x.shape[1]), -row)) for row in x])[:, :top]
    logp = np.where(ids >= 0, lp[np.arange(len(ids)), np.maximum(ids, 0)], 0.0)
    return logp, entropy[:, 0], lse[:, 0], order, np.take_along_axis(lp, order, 1), lp


def _check_rows(r, ids, top, dtype):
    x, ids = r["x"], np.asarray(ids)
    logp, entropy, lse, order, top_logp, _ = _row_reference(x, ids, top)
    # differences to the maximum that an exponential can tell from minus infinity
    near = np.minimum(np.where(np.isfinite(x), x.max(-1, keepdims=True) - x, 0.0), 104.0).max(-1)
    # sums of at most 64 terms a thread and a dozen joins, exponentials whose argument is off by `near` roundings, logarithms
    f = (96 + 4 * near) * E24
    same = lambda a, b, tol: ((np.abs(a - b) <= tol) | (a == b)).all()  # noqa: E731
    assert same(to_host(r["lse"]), lse, f + 2 * E24 * np.abs(lse))
    assert same(to_host(r["logp"]), logp, f + 4 * E24 * np.abs(logp))
    assert same(to_host(r["entropy"]), entropy, 2 * f * (1 + near))
    assert np.array_equal(r["top_ids"].cpu().numpy(), order)
    assert same(to_host(r["top_logp"]), top_logp, f[:, None] + 4 * E24 * np.abs(top_logp))


def _masked_rows(dtype, fill, rows, vocab):
    """rows masked with `fill` in the ways that programs mask: all but two tokens, everything, a block in front, every second token, together with -inf"""
    rng = np.random.default_rng(vocab + rows)
    x = (rng.normal(size=(rows, vocab)) * 3).astype(np.float32)
    fill = torch.finfo(TDT[dtype]).min if fill == "lowest" else fill
    keep = x[0, [vocab // 3, vocab - 1]]
    x[0] = fill
    x[0, [vocab // 3, vocab - 1]] = keep
    x[1] = fill
    x[2, :vocab // 2] = fill
    x[3, ::2] = fill
    x[4, : vocab - 2] = fill
    x[4, : vocab // 4] = -np.inf
    ids = rng.integers(0, vocab, rows)
    ids[:5] = [vocab - 1, 7, 3, 1, vocab - 3]     # of allowed tokens and of masked ones
    return x, ids


MASKED = [(5, 300), (600, 1000), (5, 9000), (5, 40001), (300, 40001), (5, 140000)]   # one slab, several, several rows a workgroup, split rows


@pytest.mark.parametrize("rows,vocab", MASKED)
@pytest.mark.parametrize("dtype,fill", [("fp32", -1e10), ("fp32", -1e30), ("fp32", "lowest"), ("bf16", -1e10), ("bf16", -1e30), ("bf16", "lowest"), ("fp16", "lowest"), ("fp32", -1e9), ("bf16", -1e4)])
def test_logprobs_of_masked_vocabularies(ctx, dtype, fill, rows, vocab):  # noqa: F811
    x, ids = _masked_rows(dtype, fill, rows, vocab)
    for work in (True, False):
        r = _logprobs(ctx, dtype, x, ids, 6, vocab + 3, work)
        ctx.sync()
        _check_rows(r, ids, 6, dtype)


@pytest.mark.parametrize("dtype,offset", [("fp32", 300.0), ("fp32", -1.0e4), ("fp32", 2.0e6), ("bf16", 1.0e3), ("fp16", 2.0e4)])
@pytest.mark.parametrize("rows,vocab", [(4, 2000), (3, 40001), (3, 140000)])
def test_logprobs_do_not_depend_on_a_common_offset(ctx, dtype, offset, rows, vocab):  # noqa: F811
    # log p and the entropy are functions of the differences alone, however far from zero the logits are
    rng = np.random.default_rng(vocab)
    x = (rng.normal(size=(rows, vocab)) * 3 + offset).astype(np.float32)
    ids = rng.integers(0, vocab, rows)
    r = _logprobs(ctx, dtype, x, ids, 5)
    ctx.sync()
    _check_rows(r, ids, 5, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [3, 2000, 40001, 140000])
def test_logprobs_of_rows_of_nan_are_nan(ctx, dtype, vocab):  # noqa: F811
    # a model that has diverged: nothing but NaN, or NaN where the rest is masked away; it must not pass for a row without a possible token
    x = np.random.default_rng(vocab).normal(size=(5, vocab)).astype(np.float32)
    x[1] = np.nan
    x[2] = -np.inf
    x[2, vocab // 2] = np.nan
    x[3] = -np.inf
    ids = np.array([0, 1, 2, 1, 0])
    g = torch.ones(5, device="cuda")
    for work in (True, False):
        r = _logprobs(ctx, dtype, x, ids, 2, work=work, g=g, h=g)
        ctx.sync()
        for name in ("logp", "entropy", "lse"):
            got = to_host(r[name])
            assert np.isnan(got[[1, 2]]).all() and np.isfinite(got[[0, 4]]).all(), name
        assert to_host(r["lse"])[3] == -np.inf and to_host(r["logp"])[3] == -np.inf and to_host(r["entropy"])[3] == 0 and (r["dx"][3] == 0).all()
        assert np.isnan(r["dx"][[1, 2]]).all() and np.isfinite(r["dx"][[0, 4]]).all()
        assert np.isnan(to_host(r["top_logp"])[[1, 2]]).all()
        top = r["top_ids"].cpu().numpy()
        assert ((top >= 0) & (top < vocab)).all()


@pytest.mark.parametrize("rows,vocab", [(5, 300), (5, 9001), (300, 40001), (5, 140000)])
@pytest.mark.parametrize("dtype,fill,offset", [("fp32", "lowest", 0.0), ("fp32", -1e9, 0.0), ("bf16", "lowest", 0.0), ("bf16", -1e10, 0.0), ("fp16", "lowest", 0.0), ("fp32", -1e4, 3.0e4), ("fp32", -1e4, 290.0),
                                               ("fp32", -1e4, 200.0), ("bf16", -1e4, 3.0e4), ("fp16", -6e4, -5.0e3), ("bf16", -1e4, 2.0e3)])
def test_logprob_gradients_of_masked_and_far_rows(ctx, dtype, fill, offset, rows, vocab):  # noqa: F811
    # lse alone does not hold log p of a row whose logits are all far from zero (a row of nothing but the mask is one)
    x, ids = _masked_rows(dtype, fill, rows, vocab)
    x = np.where(x > -5e3, x + np.float32(offset), x).astype(np.float32)
    g, h = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    gh, hh = to_host(g)[:, None], to_host(h)[:, None]
    for ld, in_place in ((vocab, False), (vocab + 5, True)):
        r = _logprobs(ctx, dtype, x, ids, 6, ld, True, g, h, in_place)
        ctx.sync()
        if not in_place:
            _check_rows(r, ids, 6, dtype)
            xs = r["x"]
            _, entropy, lse, _, _, lp = _row_reference(xs, ids, 0)
            p = np.exp(lp)
            ref = -p * (gh + hh * (np.where(p > 0, lp, 0.0) + entropy[:, None]))
            ref[np.arange(rows), ids] += gh[:, 0]
            near = np.minimum(np.where(np.isfinite(xs), xs.max(-1, keepdims=True) - xs, 0.0), 104.0).max(-1)
            f = (96 + 4 * near) * E24
            # what the last bit of an lse up to 256 (fp32) or 4096 (16-bit formats) leaves open in log p
            left = np.minimum(np.abs(lse), 256.0 if dtype == "fp32" else 4096.0) * E24
            size = np.abs(gh) + np.abs(hh) * (near + 2 * np.log(vocab) + 2)[:, None]
            tol = (U[dtype] + 2 * E24) * np.abs(ref) + (8 * f + 4 * left)[:, None] * p * size + LOW[dtype]
        err = np.abs(r["dx"] - ref)
        assert (err <= tol).all(), (in_place, (err / tol).max())


# ------------------------------------------------------------------------------------- what l2l_sync reports
def test_sync_names_every_kind_of_bad_input(ctx):  # noqa: F811
    x = Problem("bf16", 2, 2, 64, [40, 50], seed=8)
    plan = P.make_attention(dtype="bf16", heads=2, head_dim=64, sequences=2, max_len=50, rows=x.rows, first=dev_i32([0, x.rows - 10]), length=dev_i32([40, 50]))
    logits = torch.randn(3, 100, device="cuda")
    out = [torch.empty(3, device="cuda") for _ in range(3)]

    def sequence():
        ctx.op_attention(plan, x.q, x.q.stride(0), x.k, x.k.stride(0), x.v, x.v.stride(0), x.o, x.o.stride(0))

    def token():
        ctx.op_token_logprobs(P.L2L_F32, 3, 100, logits, 100, dev_i32([1, 100, 2]), *out)
    for calls, named, not_named in (((sequence,), "sequence that does not fit", "token id"), ((token,), "token id", "sequence that does not fit"), ((sequence, token), None, None)):
        for call in calls:
            call()
        with pytest.raises(P.L2LError) as e:
            ctx.sync()
        if named:
            assert named in str(e.value) and not_named not in str(e.value)
        else:
            assert "sequence that does not fit" in str(e.value) and "token id" in str(e.value)
        ctx.sync()


# ------------------------------------------------------------------------------------- attention
def _plan(x, causal, scale):
    return P.make_attention(dtype=x.dtype, heads=x.heads, kv_heads=x.kv, head_dim=x.d, sequences=len(x.lengths), max_len=max(x.lengths), rows=x.rows, first=dev_i32(x.first),
                            length=dev_i32(x.lengths), causal=causal, scale=scale)


def _check_large_scores(x, causal, scale):
    """o, lse, dq, dk, dv, entry by entry, where what bounds the error is the scores' own size: a sum of d products rounds d times, by up to 2^-24 of
    the products' magnitudes together each, which is an absolute error of the score and a relative one of P"""
    host = {m: to_host(getattr(x, m)) for m in ("q", "k", "v", "do", "o", "dq", "dk", "dv", "lse")}
    d, u, G, low = x.d, U[x.dtype], x.heads // x.kv, LOW[x.dtype]
    uP = 0.0 if x.dtype == "fp32" else u
    for b, n in enumerate(x.lengths):
        r = slice(x.first[b], x.first[b] + n)
        for hk in range(x.kv):
            ck = slice(hk * d, hk * d + d)
            k, v = host["k"][r, ck], host["v"][r, ck]
            total = dict(dk=0, dv=0, dk_tol=0, dv_tol=0)
            for h in range(hk * G, hk * G + G):
                c = slice(h * d, h * d + d)
                q, do = host["q"][r, c], host["do"][r, c]
                o, lse, prob = F.attention(q, k, v, scale, causal, 1.0)
                dq, dk, dv, dS = F.attention_bwd(q, k, v, scale, 1.0, prob, do)
                e = (d + 4) * E24 * scale * (np.abs(q) @ np.abs(k).T).max()      # of a score
                lse_tol = e + (n + 32 + 2 * np.abs(lse)) * E24
                assert (np.abs(host["lse"][h, r] - lse) <= lse_tol).all(), ("lse", b, h)
                f = 2 * e + (n + d + 32) * E24                                    # of P in the forward pass: its score and its row's sum
                fb = 2 * e + (n + 2 * d + 32) * E24 + (d / 2 + 4) * np.abs(lse).max() * E24      # in the backward pass: its score, lse and sums that begin at lse
                o_in = (uP + f) * (prob @ np.abs(v)) + n * low * np.abs(v).max()
                o_tol = o_in + u * (np.abs(o) + o_in) + low
                assert (np.abs(host["o"][r, c] - o) <= o_tol).all(), ("o", b, h)
                D = (np.abs(do) * np.abs(o)).sum(-1)[:, None]
                dP = np.abs(do) @ np.abs(v).T
                dS_tol = (uP + fb) * np.abs(dS) + prob * ((np.abs(do) * o_tol).sum(-1)[:, None] + fb * (dP + D)) * (1 + u) + low
                dq_tol = scale * (dS_tol @ np.abs(k)) + scale * n * E24 * (np.abs(dS) @ np.abs(k))
                dq_tol = dq_tol + u * (np.abs(dq) + dq_tol) + low
                assert (np.abs(host["dq"][r, c] - dq) <= dq_tol).all(), ("dq", b, h)
                total["dk"] += dk
                total["dv"] += dv
                total["dk_tol"] += scale * (dS_tol.T @ np.abs(q)) + scale * G * n * E24 * (np.abs(dS).T @ np.abs(q))
                total["dv_tol"] += (uP + fb + G * n * E24) * (prob.T @ np.abs(do)) + n * low * np.abs(do).max()
            for name in ("dk", "dv"):
                tol = total[name + "_tol"]
                assert (np.abs(host[name][r, ck] - total[name]) <= tol + u * (np.abs(total[name]) + tol) + low).all(), (name, b, hk)


@pytest.mark.parametrize("scale", [4.0, 64.0])
@pytest.mark.parametrize("dtype,d,lengths", [("bf16", 64, [200, 33, 2]), ("fp16", 96, [200, 33, 2]), ("fp32", 64, [200, 33, 2]), ("bf16", 128, [1300]), ("fp32", 32, [1300]), ("fp16", 64, [100, 128, 1])])
def test_attention_of_large_scores(ctx, dtype, d, lengths, scale):  # noqa: F811
    # scores of hundreds and thousands, rows that one workgroup adds up and rows in parts
    x = Problem(dtype, 2, 1, d, lengths, True, 0.0, seed=3)
    x.plan = _plan(x, True, scale)
    x.forward(ctx)
    x.backward(ctx)
    ctx.sync()
    _check_large_scores(x, True, scale)


def _means_over_the_largest(x, causal, scale):
    """q and k are whole numbers and a score is at least a thousand times the next one off: o is the mean of v over a row's largest scores"""
    o, lse, d, G = to_host(x.o), to_host(x.lse), x.d, x.heads // x.kv
    for b, n in enumerate(x.lengths):
        r = slice(x.first[b], x.first[b] + n)
        for h in range(x.heads):
            c, ck = slice(h * d, h * d + d), slice(h // G * d, h // G * d + d)
            s, v = to_host(x.q[r, c]) @ to_host(x.k[r, ck]).T, to_host(x.v[r, ck])
            if causal:
                s = np.where(np.tril(np.ones((n, n), bool)), s, -np.inf)
            top = s.max(-1)
            best = s == top[:, None]
            count = best.sum(-1)
            ref = (best @ v) / count[:, None]
            # a mean of n terms at most in fp32, then rounded to the format
            tol = U[x.dtype] * np.abs(ref) + (n + 8) * E24 * ((best @ np.abs(v)) / count[:, None]) * (1 + U[x.dtype]) + LOW[x.dtype]
            assert (np.abs(o[r, c] - ref) <= tol).all(), (causal, b, h)
            ref = scale * top + np.log(count)
            assert (np.abs(lse[h, r] - ref) <= 4 * E24 * np.abs(ref) + 8 * E24 * np.log(n + 1)).all(), (causal, b, h)


def _whole_numbers(dtype, d, lengths, amount, scale):
    """a Problem with scores that fp32 holds exactly, ties among them"""
    x = Problem(dtype, 2, 1, d, lengths, False, 0.0, seed=d + len(lengths))
    g = torch.Generator().manual_seed(d)
    mine = torch.from_numpy(x.mine).cuda()
    x.qkv[mine, :3 * d] = torch.randint(-amount, amount + 1, (sum(lengths), 3 * d), generator=g).to(TDT[dtype]).cuda()
    x.plan = _plan(x, False, scale)
    return x


def _parts_with_ties(ctx, dtype, lengths):  # noqa: F811
    x = _whole_numbers(dtype, 32, lengths, 1, 1024.0)
    assert x.work.numel() >= 2 * x.rows * 8 + 2 * 2 * x.rows * 32 * 4      # (rows in parts)
    x.forward(ctx)
    ctx.sync()
    _means_over_the_largest(x, False, 1024.0)


@pytest.mark.parametrize("lengths", [[1300], [700, 2, 901]])
def test_attention_rows_in_parts_keep_ties(ctx, lengths):  # noqa: F811
    # equal scores of some ten thousand in different parts of a row have equal weights
    _parts_with_ties(ctx, "fp32", lengths)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lengths", [[1300], [700, 2, 901]])
def test_attention_rows_in_parts_keep_ties_in_16_bits(ctx, dtype, lengths):  # noqa: F811
    _parts_with_ties(ctx, dtype, lengths)


@pytest.mark.parametrize("dtype,d,lengths", [("bf16", 64, [200, 33, 2]), ("fp16", 64, [200, 33, 2]), ("fp32", 64, [200, 33, 2]), ("bf16", 128, [1300]), ("fp16", 96, [1300]), ("fp32", 32, [1300]),
                                             ("bf16", 64, [100, 128, 1]), ("fp16", 32, [100, 128, 1]), ("fp32", 64, [60, 33, 1])])
@pytest.mark.parametrize("amount", [2, 200])
def test_attention_forward_of_scores_of_any_size(ctx, dtype, d, lengths, amount):  # noqa: F811
    # scores of up to 2^18 and 2^32; the products of a score and its scale are beyond what their last bits may be a factor of
    for causal in (False, True):
        x = _whole_numbers(dtype, d, lengths, amount, 1024.0)
        x.plan = _plan(x, causal, 1024.0)
        x.forward(ctx)
        ctx.sync()
        _means_over_the_largest(x, causal, 1024.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [90, 700])
def test_attention_forward_of_scores_far_below_zero(ctx, dtype, n):  # noqa: F811
    # every score of a row beyond -1e30: the least of them have all of the probability
    d = 64
    x = Problem(dtype, 1, 1, d, [n], False, 0.0, seed=5)
    mine = torch.arange(n, device="cuda") + x.first[0]
    step = torch.randperm(n, generator=torch.Generator().manual_seed(n)).cuda().float() // 128 + 1.0      # a few distinct sizes, so ties
    x.q[mine] = torch.full((n, d), 2.0 ** 52, device="cuda").to(TDT[dtype])
    x.k[mine] = (-(2.0 ** 52) * step)[:, None].expand(n, d).to(TDT[dtype])
    x.forward(ctx)
    ctx.sync()
    best = (step == 1).cpu().numpy()
    v = to_host(x.v[mine])
    ref = v[best].mean(0)
    tol = U[dtype] * np.abs(ref) + (n + 8) * E24 * np.abs(v[best]).mean(0) * (1 + U[dtype])
    assert (np.abs(to_host(x.o[mine]) - ref) <= tol).all()
    score = -(2.0 ** 104) * d * d ** -0.5
    assert (np.abs(to_host(x.lse[0, mine]) - score) <= 4 * E24 * abs(score)).all()


@pytest.mark.parametrize("p", [0.0, 0.2])
@pytest.mark.parametrize("d,causal,size", [(64, False, 1e-3), (64, True, 1e-4), (96, False, 1e-4), (32, True, 1e-3), (128, False, 1e-3), (64, False, 30.0)])
def test_attention_fp16_gradients_of_any_size(ctx, d, causal, size, p):  # noqa: F811
    """Long rows spread a gradient over many keys: dS is smaller than dO by the length and may lie below fp16's normal range where its
    sums over keys or queries do not.  Against fp64, what the results' own rounding leaves and a few half steps of P and dS."""
    n, heads = 3000, 2
    x = Problem("fp16", heads, 1, d, [n], causal, p, seed=d)
    mine = slice(x.first[0], x.first[0] + n)
    x.do[mine] = (x.do[mine].float() * size).half()
    x.forward(ctx)
    x.backward(ctx)
    ctx.sync()
    k, v, scale = to_host(x.k[mine]), to_host(x.v[mine]), d ** -0.5
    dk, dv, parts = 0, 0, []
    for h in range(heads):
        c = slice(h * d, h * d + d)
        Z = F.drop_factors_attention(n, h, p, SEED, SITE)
        _, _, prob = F.attention(to_host(x.q[mine, c]), k, v, scale, causal, Z)
        dq, dk1, dv1, _ = F.attention_bwd(to_host(x.q[mine, c]), k, v, scale, Z, prob, to_host(x.do[mine, c]))
        dk, dv = dk + dk1, dv + dv1
        parts.append(("dq", to_host(x.dq[mine, c]), dq))
    for name, got, ref in parts + [("dk", to_host(x.dk[mine]), dk), ("dv", to_host(x.dv[mine]), dv)]:
        own = np.linalg.norm(ref.astype(np.float16).astype(np.float64) - ref)
        assert np.linalg.norm(got - ref) <= own + 4 * U["fp16"] * np.linalg.norm(ref), (name, np.linalg.norm(got - ref) / np.linalg.norm(ref), own / np.linalg.norm(ref))


@pytest.mark.parametrize("d,causal", [(64, False), (96, True)])
def test_attention_fp16_gradients_of_rows_of_different_sizes(ctx, d, causal):  # noqa: F811
    # no gradient at first, then large ones, one of them by far: what the first rows allow must not overflow at the later ones
    n = 1000
    x = Problem("fp16", 2, 1, d, [n], causal, 0.0, seed=d, amp=1.5)
    size = torch.zeros(n, 1, device="cuda")
    size[400:] = 20.0
    size[700] = 600.0
    mine = slice(x.first[0], x.first[0] + n)
    x.do[mine] = (x.do[mine].float() * size).half()
    x.forward(ctx)
    x.backward(ctx)
    ctx.sync()
    x.check()


def test_attention_fp16_backward_gives_the_same_bits_captured_and_in_any_workspace():
    # what the dQ kernel leaves for the dK / dV kernel is written anew by every call
    stream = torch.cuda.Stream()
    c = P.Context(P.make_config(64, 2, 128, 16, 2, 2, "bf16", 1e-5, 0), stream.cuda_stream, stream.cuda_stream)
    try:
        for lengths in ([300, 257, 64, 1], [1500]):
            x = Problem("fp16", 4, 2, 64, lengths, True, 0.1, seed=6)
            outs = (x.o, x.lse, x.dq, x.dk, x.dv)

            def both():
                x.forward(c)
                x.backward(c)
            torch.cuda.synchronize()
            both()
            torch.cuda.synchronize()
            eager = [t.clone() for t in outs]
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                both()
            for fill in (255, 0, 127):
                for t in outs:
                    t.fill_(7.0)
                x.work.fill_(fill)
                torch.cuda.synchronize()
                with torch.cuda.stream(stream):
                    graph.replay()
                torch.cuda.synchronize()
                torch.randn(1000, device="cuda").sum().item()
                assert all(torch.equal(a, b) for a, b in zip(outs, eager))
            x.check()
    finally:
        c.close()


def test_attention_in_parts_without_lse(ctx):  # noqa: F811
    for dtype in ("bf16", "fp32"):
        x = Problem(dtype, 2, 1, 64, [1100, 300], False, 0.0, seed=12)
        x.forward(ctx)
        ctx.sync()
        o = x.o.clone()
        x.o.fill_(7.0)
        ctx.op_attention(x.plan, x.q, x.q.stride(0), x.k, x.k.stride(0), x.v, x.v.stride(0), x.o, x.o.stride(0), None, x.work)
        ctx.sync()
        assert torch.equal(x.o, o)
