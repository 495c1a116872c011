"""od_token_logprobs and od_token_logprobs_grad against the definitions in 64 bits.

Tolerances. Every number is held in fp32 (half a step: 2^-24). A term exp2((x - M) c) has the error of
its argument (three roundings: 3 * 2^-24 |(x - M) / T|) and of ex2.approx (2^-22); a thread's sum is raised
to a new maximum at most a few times (2^-22 each) and the terms of a row are added in chains of at most a few
dozen (2^-24 each). Where a term counts at all in a sum |(x - M) / T| is below 20, so that a row sum is
within 2^-17 of its value, its logarithm within 2^-17 too, and the log probability adds two roundings of
(x_t - M) / T and one of the result. The gradient's terms p (G + g (ln p + H)) have the relative error of p, which
grows with |(x - M) / T|; a bf16 gradient is rounded once more (2^-8).
"""
import math

import numpy as np
import pytest
import torch

from paper_2507_02659_b200 import binding as od

pytestmark = pytest.mark.gpu

E = 2.0 ** -17
INF = math.inf


@pytest.fixture(scope="module")
def ctx(cuda_device):
    torch.cuda.set_device(cuda_device)
    c = od.Context(cuda_device, 10, 10, 1, 1)               # (no vocabulary map, a batch of one: neither is needed)
    yield c
    c.close()


def padded(x, fill=float("nan")):
    """The same rows with strides of whole 16 bytes; what lies behind a row is NaN."""
    B, R, V = x.shape
    per = 16 // x.element_size()
    store = torch.full((B, R, (V // per + 2) * per), fill, dtype=x.dtype, device=x.device)
    store[:, :, :V] = x
    return store[:, :, :V]


def make(B, R, V, dtype, seed, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(B, R, V, generator=g, device="cuda") * spread
    ids = torch.randint(-1, V, (B, R), generator=g, device="cuda", dtype=torch.int32)
    T = torch.tensor([1.0, 0.7, 0.5, 2.0], device="cuda").repeat(-(-B // 4))[:B].contiguous()
    return padded(x.to(dtype)), ids, T


def reference(x, ids, T, n):
    """The definitions in 64 bits, a row at a time on the host's numpy order rules: dict of float64 tensors."""
    B, R, V = x.shape
    d = x.double()
    M = d.max(2, keepdim=True).values
    z = torch.where(d == M, 0.0, (d - M) / T.double()[:, None, None])
    e = torch.exp(z)
    S = e.sum(2, keepdim=True)
    ln = torch.log(S)
    lp = z - ln
    mean = (e * torch.where(e > 0, z, 0.0)).sum(2) / S.squeeze(2)
    at = torch.gather(lp, 2, ids.long().clamp(0, V - 1)[:, :, None]).squeeze(2)
    has = (ids >= 0) & (ids < V)
    out = dict(logprob=torch.where(has, at, 0.0), entropy=ln.squeeze(2) - mean, row_max=M.squeeze(2), row_sum=S.squeeze(2),
               lp=lp, z=z, mean=mean)
    if n:
        order = torch.sort(d, dim=2, descending=True, stable=True).indices[:, :, :n]
        value = torch.gather(lp, 2, order)
        top = torch.where(value > -INF, order, -1)
        out["top_ids"] = torch.nn.functional.pad(top, (0, n - top.shape[2]), value=-1)
        out["top_logprobs"] = torch.nn.functional.pad(value, (0, n - value.shape[2]), value=-INF)
    return out


def same(got, want, tol):
    got, want = got.double(), want.double()
    want = torch.where(want.abs() >= 2.0 ** 128, want.sign() * INF, want)    # beyond fp32
    tol = torch.as_tensor(tol, dtype=torch.float64, device=got.device).expand_as(want)
    exact = got == want                                     # infinities too
    bad = ~(exact | ((got - want).abs() <= tol))
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}: {got[bad][:4].tolist()} for {want[bad][:4].tolist()}, tolerance {tol[bad][:4].tolist()}"


def relative(lp):
    return E + 2.0 ** -22 * torch.where(torch.isfinite(lp), lp.abs(), 0.0)


def check(out, ref, n):
    assert torch.equal(out.row_max.double(), ref["row_max"])
    same(out.row_sum, ref["row_sum"], E * ref["row_sum"])
    same(out.logprob, ref["logprob"], relative(ref["logprob"]))
    same(out.entropy, ref["entropy"], E * (1 + ref["mean"].abs()) + 2.0 ** -22 * ref["row_sum"].log())
    if n:
        assert torch.equal(out.top_ids.long(), ref["top_ids"])
        same(out.top_logprobs, ref["top_logprobs"], relative(ref["top_logprobs"]))


SHAPES = [(1, 1, 1, 1), (1, 1, 7, 32), (2, 3, 255, 5), (3, 2, 1000, 32), (2, 5, 8193, 20), (1, 2, 100277, 3), (5, 2, 32000, 0),
          (300, 1, 4099, 4), (1, 1, 152064, 20), (2, 1, 16, 16), (37, 9, 20011, 8), (4, 7, 65536, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,R,V,n", SHAPES)
def test_scores(ctx, B, R, V, n, dtype):
    x, ids, T = make(B, R, V, dtype, 1)
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=n)
    check(out, reference(x, ids, T, n), n)
    assert not out.flags.any()


def grad_reference(x, ids, T, ref, g_lp, g_h, g_top, n):
    B, R, V = x.shape
    Td = T.double()[:, None, None]
    p = torch.exp(ref["lp"])
    has = (ids >= 0) & (ids < V)
    G = torch.zeros(B, R, dtype=torch.float64, device=x.device)
    spike = torch.zeros(B, R, V, dtype=torch.float64, device=x.device)
    absg = spike.clone()
    for idx, g in ([] if g_lp is None else [(torch.where(has, ids.long(), -1)[:, :, None], g_lp[:, :, None])]) + \
                  ([] if g_top is None else [(ref["top_ids"], g_top)]):
        w = torch.where(idx >= 0, g.double(), 0.0)
        G += w.sum(2)
        spike.scatter_add_(2, idx.clamp(min=0), w)
        absg.scatter_add_(2, idx.clamp(min=0), w.abs())
    inner = torch.where(p > 0, ref["lp"], 0.0) + ref["entropy"][:, :, None]
    gh = g_h.double()[:, :, None] if g_h is not None else 0.0
    v = (spike - p * (G[:, :, None] + gh * inner)) / Td
    # a sum of n + 1 weights; p's relative error; one rounding of each product
    size = p * ((n + 2) * G.abs()[:, :, None] + absg.sum(2, keepdim=True)
                + (abs(gh) if g_h is None else gh.abs()) * (ref["lp"].clamp(min=-1e30).abs() + ref["entropy"][:, :, None] + 1))
    tol = (size * (E + ref["z"].clamp(min=-1e30).abs() * 2.0 ** -21) + absg * 2.0 ** -20) / Td + 1e-30
    return v, tol


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,R,V,n", SHAPES)
def test_gradient(ctx, B, R, V, n, dtype):
    x, ids, T = make(B, R, V, dtype, 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    g_lp = torch.randn(B, R, generator=g, device="cuda")
    g_h = torch.randn(B, R, generator=g, device="cuda")
    g_top = torch.randn(B, R, n, generator=g, device="cuda") if n else None
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=n)
    ref = reference(x, ids, T, n)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for a, b, c in [(g_lp, g_h, g_top), (g_lp, None, None), (None, g_h, None), (None, None, g_top), (None, None, None)]:
        want, tol = grad_reference(x, ids, T, ref, a, b, c, n)
        got = od.od_token_logprobs_grad(ctx, x, ids, out, a, b, c, temperature=T)
        same(got, want, tol + half * (want.abs() + tol))
        inplace = padded(x)
        assert od.od_token_logprobs_grad(ctx, inplace, ids, out, a, b, c, temperature=T, grad=inplace) is inplace
        assert torch.equal(got, inplace)


def test_gradient_against_differences(ctx):
    """The gradient of a loss on everything that is returned against central differences of the library's own scores."""
    B, R, V, n = 2, 2, 40, 3
    x, ids, T = make(B, R, V, torch.float32, 5)
    ids.clamp_(min=0)
    g = torch.Generator(device="cuda").manual_seed(6)
    for b in range(B):                                      # logits a quarter apart: the alternatives keep their order
        for r in range(R):
            x[b, r] = torch.randperm(V, generator=g, device="cuda") / 4.0 - 5.0
    g_lp, g_h = torch.randn(B, R, generator=g, device="cuda"), torch.randn(B, R, generator=g, device="cuda")
    g_top = torch.randn(B, R, n, generator=g, device="cuda")
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=n)
    grad = od.od_token_logprobs_grad(ctx, x, ids, out, g_lp, g_h, g_top, temperature=T)
    step = 2.0 ** -6

    def loss(y):
        o = od.od_token_logprobs(ctx, y, ids, T, n_top=n)
        assert torch.equal(o.top_ids, out.top_ids)
        return (g_lp.double() * o.logprob.double()).sum() + (g_h.double() * o.entropy.double()).sum() \
            + (g_top.double() * o.top_logprobs.double()).sum()
    weights = float(g_lp.abs().sum() + g_h.abs().sum() + g_top.abs().sum())
    for b, r, t in [(0, 0, int(ids[0, 0])), (0, 1, 3), (1, 0, int(out.top_ids[1, 0, 1])), (1, 1, 39), (0, 0, 17)]:
        y = padded(x)
        y[b, r, t] += step
        up = loss(y)
        y[b, r, t] -= 2 * step
        down = loss(y)
        # the scores' error over the step, and a sixth of the third derivative (below 48, (|ln p| + H) / T^3, a weight)
        tol = weights * (4 * E / step + step ** 2 * 8)
        assert abs(float(up - down) / (2 * step) - float(grad[b, r, t])) <= tol


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [5, 777, 40000])
def test_rows_at_the_limits(ctx, V, dtype):
    """Masks of -inf and of the type's lowest value, equal logits, signed zeros, far apart values, nothing left."""
    low = torch.finfo(dtype).min
    g = torch.Generator(device="cuda").manual_seed(7)
    rows = [torch.zeros(V), torch.full((V,), -INF), torch.full((V,), low), torch.randn(V), torch.randn(V), torch.randn(V) * 1e30,
            torch.zeros(V), torch.full((V,), low), torch.full((V,), 3.0), torch.randn(V) * 50 + 1000]
    rows[3][1:] = -INF                                      # one id left
    rows[4][: V // 2] = low                                 # a mask of the lowest value
    rows[6][::2] = -0.0                                     # -0 equals 0
    rows[7][V // 2] = -INF
    rows[8][V - 1] = 4.0
    x = padded(torch.stack(rows).to(dtype)[None].cuda())
    R, n = len(rows), 4
    ids = torch.randint(0, V, (1, R), generator=g, device="cuda", dtype=torch.int32)
    ids[0, 3], ids[0, 4] = 0, V - 1
    T = torch.tensor([0.5], device="cuda")
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=n)
    keep = [i for i in range(R) if i != 1]
    ref = reference(x[:, keep], ids[:, keep], T, n)
    sub = od.LogprobOut(*(t[:, keep] for t in vars(out).values()))
    check(sub, ref, n)
    assert out.flags[0].tolist() == [0, od.OD_LF_NO_MASS] + [0] * (R - 2)
    # the row of nothing but -inf
    assert float(out.row_max[0, 1]) == -INF and float(out.row_sum[0, 1]) == 0 and float(out.entropy[0, 1]) == 0
    assert float(out.logprob[0, 1]) == -INF
    assert out.top_ids[0, 1].tolist() == [-1] * n and out.top_logprobs[0, 1].tolist() == [-INF] * n
    g_lp, g_h = torch.ones(1, R, device="cuda"), torch.ones(1, R, device="cuda")
    g_top = torch.ones(1, R, n, device="cuda")
    grad = od.od_token_logprobs_grad(ctx, x, ids, out, g_lp, g_h, g_top, temperature=T)
    want, tol = grad_reference(x[:, keep], ids[:, keep], T, ref, g_lp[:, keep], g_h[:, keep], g_top[:, keep], n)
    same(grad[:, keep], want, tol + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * (want.abs() + tol))
    assert not grad[0, 1].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_hold_nan_or_infinity(ctx, dtype):
    for V in (9, 5000, 70001):
        x = torch.randn(4, 1, V, device="cuda")
        x[0, 0, V - 1] = float("nan")
        x[1, 0, 0] = INF
        x[2, 0, V // 2] = float("nan")
        x = padded(x.to(dtype))
        ids = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
        out = od.od_token_logprobs(ctx, x, ids, n_top=2)
        assert out.flags.view(-1).tolist() == [od.OD_LF_NONFINITE] * 3 + [0]
        for t in (out.logprob, out.entropy, out.row_max, out.row_sum):
            assert torch.isnan(t[:3]).all() and torch.isfinite(t[3:]).all()
        assert (out.top_ids[:3] == -1).all() and torch.isnan(out.top_logprobs[:3]).all()
        one = torch.ones(4, 1, device="cuda")
        grad = od.od_token_logprobs_grad(ctx, x, ids, out, one, one)
        assert torch.isnan(grad[:3]).all() and torch.isfinite(grad[3:]).all()


def test_bad_temperatures_and_ids(ctx):
    V, n = 300, 2
    x, _, _ = make(7, 1, V, torch.float32, 8)
    T = torch.tensor([0.0, -1.0, float("nan"), INF, 1e-45, 1.0, 1.0], device="cuda")
    ids = torch.tensor([[1], [2], [3], [V], [4], [-7], [V]], dtype=torch.int32, device="cuda")
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=n)
    bad = od.OD_LF_BAD_TEMPERATURE
    assert out.flags.view(-1).tolist() == [bad] * 3 + [bad | od.OD_LF_BAD_ID, bad] + [od.OD_LF_BAD_ID] * 2
    for t in (out.logprob, out.entropy, out.row_max, out.row_sum):
        assert not t[:5].any()
    assert (out.top_ids[:5] == -1).all() and (out.top_logprobs[:5] == -INF).all()
    assert not out.logprob[5:].any() and (out.entropy[5:] > 0).all()
    one = torch.ones(7, 1, device="cuda")
    grad = od.od_token_logprobs_grad(ctx, x, ids, out, one, one, temperature=T)
    assert not grad[:5].any() and grad[5:].any()
    want, tol = grad_reference(x[5:], ids[5:], T[5:], reference(x[5:], ids[5:], T[5:], 0), one[5:], one[5:], None, 0)
    same(grad[5:], want, 2 * tol)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_largest_logits_in_one_threads_elements(ctx, dtype):
    """More candidates than are ranked by counting: every element that one thread reads is among the largest."""
    V, n = 152064, 32
    per = 8 if dtype == torch.bfloat16 else 4
    for rows, split in ((300, 1), (1, 8)):
        x = torch.randn(rows, 1, V, device="cuda")
        first = (V // per) // split * 3 if split > 1 else 0
        i = torch.arange(V, device="cuda") // per - first
        x[:, 0, (i >= 0) & (i % 256 < 2) & (i < 12800)] += 20.0
        x = padded(x.to(dtype))
        ids = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
        T = torch.ones(rows, device="cuda")
        out = od.od_token_logprobs(ctx, x, ids, T, n_top=n)
        for b in {0, rows - 1}:
            ref = reference(x[b:b + 1], ids[b:b + 1], T[b:b + 1], n)
            check(od.LogprobOut(*(t[b:b + 1] for t in vars(out).values())), ref, n)


def test_rows_that_do_not_count_stay_as_they_are(ctx):
    B, R, V, n = 4, 5, 1000, 3
    x, ids, T = make(B, R, V, torch.bfloat16, 9)
    n_rows = torch.tensor([0, 5, 2, 9], dtype=torch.int32, device="cuda")
    dead = torch.arange(R, device="cuda")[None] >= n_rows[:, None]
    whole = x.clone()
    x[dead] = float("nan")
    out = od.alloc_logprob_out(ctx, B, R, n)
    for t in vars(out).values():
        t.fill_(77)
    od.od_token_logprobs(ctx, x, ids, T, n_rows, n, out)
    for name, t in vars(out).items():
        assert (t[dead] == 77).all(), name
    live = ~dead
    ref = reference(whole, ids, T, n)
    sub = od.LogprobOut(*(t[live][None] for t in vars(out).values()))
    check(sub, {k: v[live][None] for k, v in ref.items()}, n)
    one = torch.ones(B, R, device="cuda")
    store = torch.full((B, R + 1, 1024), 55.0, dtype=x.dtype, device="cuda")
    grad = od.od_token_logprobs_grad(ctx, x, ids, out, one, one, torch.ones(B, R, n, device="cuda"), T, n_rows, grad=store[:, :R, :V])
    assert not grad[dead].any() and torch.isfinite(grad).all()
    assert (store[:, R] == 55).all() and (store[:, :, V:] == 55).all()


def test_ids_that_are_named_twice(ctx):
    """The given token among the alternatives, and a list of the caller's own that repeats an id."""
    V, n = 500, 4
    x, _, T = make(1, 1, V, torch.float32, 10)
    out = od.od_token_logprobs(ctx, x, None, T, n_top=n)
    assert not out.logprob.any()
    ids = out.top_ids[:, :, 2].contiguous()
    g_lp, g_top = torch.tensor([[2.0]], device="cuda"), torch.tensor([[[1.0, 3.0, 5.0, 7.0]]], device="cuda")
    ref = reference(x, ids, T, n)
    want, tol = grad_reference(x, ids, T, ref, g_lp, None, g_top, n)
    same(od.od_token_logprobs_grad(ctx, x, ids, out, g_lp, None, g_top, T), want, 2 * tol)
    out.top_ids[0, 0] = torch.tensor([9, 9, V, 9], device="cuda")    # (V: no id, it takes no part)
    ref["top_ids"] = torch.tensor([[[9, 9, -1, 9]]], device="cuda")
    want, tol = grad_reference(x, ids, T, ref, g_lp, None, g_top, n)
    same(od.od_token_logprobs_grad(ctx, x, ids, out, g_lp, None, g_top, T), want, 2 * tol)


def test_strides_and_offsets_past_32_bits(ctx):
    V, far = 1000, (1 << 31) + 8 * 1111
    store = torch.empty(far + 8192, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(store, (2, 3, V), (far, 2048, 1))
    y, ids, T = make(2, 3, V, torch.bfloat16, 11)
    x.copy_(y)
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=5)
    ref = reference(y, ids, T, 5)
    check(out, ref, 5)
    one = torch.ones(2, 3, device="cuda")
    a = od.od_token_logprobs_grad(ctx, y, ids, out, one, one, temperature=T)
    assert torch.equal(od.od_token_logprobs_grad(ctx, x, ids, out, one, one, temperature=T, grad=x), a)


def test_captured_and_replayed_on_other_inputs_and_on_another_stream(ctx):
    B, R, V, n = 3, 4, 30011, 6
    x, ids, T = make(B, R, V, torch.bfloat16, 12)
    one = torch.ones(B, R, device="cuda")
    out = od.alloc_logprob_out(ctx, B, R, n)
    grad = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        od.od_token_logprobs(ctx, x, ids, T, n_top=n, out=out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            od.od_token_logprobs(ctx, x, ids, T, n_top=n, out=out)
            od.od_token_logprobs_grad(ctx, x, ids, out, one, one, temperature=T, grad=grad)
        y, ids2, _ = make(B, R, V, torch.bfloat16, 13)
        x.copy_(y); ids.copy_(ids2)
        graph.replay()
    torch.cuda.synchronize()
    check(out, reference(y, ids2, T, n), n)
    again = od.od_token_logprobs_grad(ctx, y, ids2, out, one, one, temperature=T)
    assert torch.equal(again, grad)


def test_scores_of_a_step(ctx):
    """Beside a verification step: od_verify's row statistics are the scores' own, and serve the gradient as they are."""
    from paper_2507_02659_b200 import synth
    import parity
    w = synth.Workload("score", B=6, steps=1, k_max=4, k_min=1, v_q=1200, v_p=5003, logit_dtype="bf16", map_kind="random",
                       mapped_frac=0.7, cache_entries=100, hit_prob=0.3, logit_kind="corr", rho=0.95, temperatures=(1.0, 0.5),
                       per_seq_seed=True, gen_seed=0x5C0, unmapped_shift=2.0, sigma=2.0)
    st = synth.make_static(w)
    c = parity.make_context(w, st, "cuda:0")
    s = synth.make_step(w, st, 0, device="cuda:0")
    logits = parity.pad_rows(s.logits)
    mp, vo, so = od.od_step(c, s.draft_ids, s.draft_len, s.q_sel, s.q_rows, logits, s.temperature, s.seed, 0)
    K = w.k_max
    # the verified tokens of rows 0..m-1, the extra token at the row it was drawn from
    r = torch.arange(K + 1, device="cuda")[None]
    ids = torch.cat([mp.tgt_ids, torch.full((w.B, 1), -1, dtype=torch.int32, device="cuda")], 1)
    ids = torch.where(r < vo.n_accepted[:, None], ids, torch.where(r == vo.n_accepted[:, None], so.out_token[:, None], -1))
    n_rows = (vo.n_accepted + 1).int()
    out = od.od_token_logprobs(c, logits, ids.contiguous(), s.temperature, n_rows, 3)
    ref = reference(logits, ids, s.temperature, 3)
    live = r < n_rows[:, None]
    check(od.LogprobOut(*(t[live][None] for t in vars(out).values())), {k: v[live][None] for k, v in ref.items()}, 3)
    assert torch.equal(out.row_max[live], vo.row_max[live])
    same(out.row_sum[live], vo.row_sum[live], 4 * E * vo.row_sum[live].double())
    one = torch.ones(w.B, K + 1, device="cuda")
    from_verify = od.LogprobOut(out.logprob, out.entropy, vo.row_max, vo.row_sum, out.top_ids, out.top_logprobs, out.flags)
    grad = od.od_token_logprobs_grad(c, logits, ids.contiguous(), from_verify, one, one, temperature=s.temperature, n_rows=n_rows)
    want, tol = grad_reference(logits, ids, s.temperature, ref, one, one, None, 0)
    same(grad[live], want[live], 8 * tol[live] + 2.0 ** -8 * want[live].abs())
    assert not grad[~live].any()
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,V", [(1, 32000), (1, 7), (3, 152064), (500, 4099)])
def test_rows_with_nearly_all_mass_on_one_token(ctx, rows, V, dtype):
    """Entropies and log probabilities near zero keep their digits: they are sums of the other terms alone, each within
    2^-22 + 3 * 2^-24 |(x - M) / T| of its value, below 2^-16 with |(x - M) / T| up to 70, and of their products with that."""
    g = torch.Generator(device="cuda").manual_seed(18)
    x = torch.randn(rows, 1, V, generator=g, device="cuda")
    at = torch.randint(0, V, (rows,), generator=g, device="cuda")
    x[torch.arange(rows), 0, at] = 14.0 + 12.0 * torch.rand(rows, generator=g, device="cuda")
    x = padded(x.to(dtype))
    T = torch.full((rows,), 0.7, device="cuda")
    ids = at.int()[:, None]
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=1)
    ref = reference(x, ids, T, 1)
    d = torch.where(ref["z"] == 0, -torch.inf, ref["z"])    # without the largest
    rest = torch.exp(d).sum(2)
    less = -(torch.exp(d) * torch.where(d > -torch.inf, d, 0.0)).sum(2)
    want_h = torch.log1p(rest) + less / (1 + rest)
    assert torch.equal(out.top_ids[:, :, 0].long(), at[:, None])
    same(out.logprob, -torch.log1p(rest), 2.0 ** -16 * rest)
    same(out.top_logprobs[:, :, 0], -torch.log1p(rest), 2.0 ** -16 * rest)
    same(out.entropy, want_h, 2.0 ** -15 * want_h)
    same(out.row_sum, 1 + rest, E * (1 + rest))


def test_long_rows_of_many(ctx):
    """A block to a row and more turns of a thread than it leaves maxima."""
    B, V, n = 300, 300007, 20
    x, ids, T = make(B, 1, V, torch.bfloat16, 15)
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=n)
    for lo in (0, B - 8):
        ref = reference(x[lo:lo + 8], ids[lo:lo + 8], T[lo:lo + 8], n)
        check(od.LogprobOut(*(t[lo:lo + 8] for t in vars(out).values())), ref, n)


def test_two_streams_at_once(ctx):
    """No scratch: calls on one context need no order."""
    cases = [make(b, r, v, torch.bfloat16, 16) for b, r, v in ((1, 1, 152064), (40, 4, 32000))]
    want = [vars(od.od_token_logprobs(ctx, x, ids, T, n_top=7)) for x, ids, T in cases]
    outs = [od.alloc_logprob_out(ctx, x.shape[0], x.shape[1], 7) for x, _, _ in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for (x, ids, T), out, s in zip(cases, outs, streams):
            with torch.cuda.stream(s):
                od.od_token_logprobs(ctx, x, ids, T, n_top=7, out=out)
    torch.cuda.synchronize()
    for w, out in zip(want, outs):
        assert all(torch.equal(w[k], t) for k, t in vars(out).items())


def test_with_and_without_the_extension(ctx, monkeypatch):
    x, ids, T = make(3, 4, 777, torch.float32, 17)
    n_rows = torch.tensor([1, 4, 2], dtype=torch.int32, device="cuda")
    one, g_top = torch.ones(3, 4, device="cuda"), torch.ones(3, 4, 5, device="cuda")

    def both():
        out = od.od_token_logprobs(ctx, x, ids, T, n_rows, 5, out=od.alloc_logprob_out(ctx, 3, 4, 5))
        return [*vars(out).values(), od.od_token_logprobs_grad(ctx, x, ids, out, one, one, g_top, T, n_rows, grad=padded(x))]
    a = both()
    monkeypatch.setattr(od, "_native", od._InPython())
    assert all(torch.equal(p, q) for p, q in zip(a, both()))


def test_refusals(ctx):
    x, ids, T = make(2, 3, 64, torch.bfloat16, 14)
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=2)
    with pytest.raises(TypeError):
        od.od_token_logprobs(ctx, x.half(), ids, T)
    with pytest.raises(TypeError):
        od.od_token_logprobs(ctx, x, ids.long(), T)
    with pytest.raises(ValueError):
        od.od_token_logprobs(ctx, x, ids[:1], T)
    with pytest.raises(ValueError):
        od.od_token_logprobs(ctx, x.transpose(1, 2), None, T)
    with pytest.raises(ValueError):
        od.od_token_logprobs(ctx, x, ids, T, n_top=3, out=out)
    with pytest.raises(ValueError):
        od.od_token_logprobs(ctx, x.cpu(), ids, T)
    with pytest.raises(od.OdError) as e:
        od.od_token_logprobs(ctx, x, ids, T, n_top=33)
    assert e.value.status == od.OD_ERR_INVALID_ARG
    odd = torch.zeros(2, 3, 65, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(od.OdError) as e:
        od.od_token_logprobs(ctx, odd, ids, T)
    assert e.value.status == od.OD_ERR_ALIGNMENT
    with pytest.raises(od.OdError) as e:                    # broadcast rows overlap
        od.od_token_logprobs(ctx, x[:1].expand(2, 3, 64), ids, T)
    assert e.value.status == od.OD_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        od.od_token_logprobs_grad(ctx, x, ids, out, out.logprob, grad=torch.empty(2, 3, 64, device="cuda"))
    with pytest.raises(ValueError):
        od.od_token_logprobs_grad(ctx, x, ids, out, out.logprob, g_top=torch.zeros(2, 3, 5, device="cuda"))
    with pytest.raises(ValueError):                         # rows without sequences
        od.od_token_logprobs(ctx, x[0], ids[:1], T[:1], n_top=2, out=od.alloc_logprob_out(ctx, 1, 3, 2))
    assert od.od_token_logprobs(ctx, x[:0], ids[:0], T[:0], n_top=2).logprob.shape == (0, 3)
    np.testing.assert_array_equal(od.od_token_logprobs(ctx, x, ids, T, n_top=2).top_ids.cpu(), out.top_ids.cpu())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [0, 4])
@pytest.mark.parametrize("rows,V", [(1, 40), (1, 152064), (40, 152064), (100, 152064), (200, 60000), (400, 130001), (700, 4099), (1300, 300)])
def test_rows_with_nearly_all_mass_on_one_token_are_the_same_in_every_run(ctx, rows, V, n, dtype):
    """Every warp of a block decides by the same sums that one token has nearly all of the mass, whichever of them holds it: one to
    eight blocks a row, of either size, with such rows beside ordinary ones. The bounds of the test above."""
    g = torch.Generator(device="cuda").manual_seed(19)
    x = torch.randn(rows, 1, V, generator=g, device="cuda")
    at = torch.randint(0, V, (rows,), generator=g, device="cuda")
    peak = torch.arange(rows, device="cuda") % 4 != 3
    x[torch.arange(rows), 0, at] = torch.where(peak, 16.0 + 10.0 * torch.rand(rows, generator=g, device="cuda"), 1.0)
    x = padded(x.to(dtype))
    T = torch.full((rows,), 0.7, device="cuda")
    ids = at.int()[:, None]
    first = vars(od.od_token_logprobs(ctx, x, ids, T, n_top=n))
    z = ((x.double() - x.double().max(2, keepdim=True).values) / T.double()[:, None, None]).squeeze(1)[peak]
    rest = torch.exp(torch.where(z == 0, -INF, z)).sum(1)
    assert torch.equal(z.argmax(1), at[peak])
    same(first["logprob"][peak, 0], -torch.log1p(rest), 2.0 ** -16 * rest)
    for _ in range(30):
        again = vars(od.od_token_logprobs(ctx, x, ids, T, n_top=n))
        assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,V", [(4, 33), (40, 32000), (300, 4099)])
def test_gradients_of_rows_with_nearly_all_mass_on_one_token(ctx, rows, V, dtype):
    """At that token within 2^-21 of the weights' magnitudes, as the header says: the row sum, its product with T, the quotient, two
    products, sum / T and the difference are a rounding of 2^-24 each (of G + g_entropy (entropy - ln row_sum), where the
    logarithm has 2^-23 of row_sum's own too, and entropies are below 0.01 here); elsewhere relative to p (G + g_entropy (ln p + entropy))."""
    g = torch.Generator(device="cuda").manual_seed(20)
    x = torch.randn(rows, 1, V, generator=g, device="cuda")
    at = torch.randint(0, V, (rows,), generator=g, device="cuda")
    x[torch.arange(rows), 0, at] = 16.0 + 10.0 * torch.rand(rows, generator=g, device="cuda")
    x = padded(x.to(dtype))
    T = torch.full((rows,), 0.7, device="cuda")
    ids = at.int()[:, None]
    ids[1::4] = (ids[1::4] + 1) % V                         # another token than the one with the mass
    g_lp, g_h = torch.randn(rows, 1, generator=g, device="cuda"), torch.randn(rows, 1, generator=g, device="cuda")
    g_top = torch.randn(rows, 1, 2, generator=g, device="cuda")
    out = od.od_token_logprobs(ctx, x, ids, T, n_top=2)
    ref = reference(x, ids, T, 2)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for a, b, c in [(g_lp, None, None), (g_lp, g_h, g_top), (None, g_h, None)]:
        want, tol = grad_reference(x, ids, T, ref, a, b, c, 2)
        weights = sum(t.double().abs().sum(2) if t.dim() == 3 else t.double().abs() for t in (a, b, c) if t is not None)
        limit = (2.0 ** -21 * weights / T.double()[:, None])[:, :, None].expand_as(want)
        named = torch.zeros_like(want, dtype=torch.bool).scatter_(2, at[:, None, None], True)
        named.scatter_(2, ids.long()[:, :, None], True).scatter_(2, ref["top_ids"], True)
        tol = torch.where(named, limit, tol)
        same(od.od_token_logprobs_grad(ctx, x, ids, out, a, b, c, temperature=T), want, tol + half * (want.abs() + tol))
