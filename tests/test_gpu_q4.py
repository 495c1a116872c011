"""od_q4_logits and od_q4_logits_grad against products in 64 bits.

Tolerances. A product of an input and a code is exact (an fp32 input is taken in three bf16 pieces, a scaled bf16 one in
two), so the errors are those of fp32 sums: a matrix instruction adds sixteen products to its accumulator with an
error of at most 2^-22 of the largest sum of magnitudes it meets, an fp32 step 2^-24. The instructions add x u, the 8 that is
to be taken off a code is in what a group's sum begins at: the magnitudes are those of x u s and 8 x s, S = sum |x s| (u + 8).
A logit goes through group / 16 * 3 instructions per group and one step per group, its group's beginning through
group / 8 + 2 fp32 steps; a gradient through at most vocab / 16 * 3 instructions, one rounding of each scaled input, and the
steps that join the parts (below 64). The result is rounded once to its type.
"""
import math

import pytest
import torch

from paper_2507_02659_b200 import binding as od

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


@pytest.fixture(scope="module")
def ctx(cuda_device):
    torch.cuda.set_device(cuda_device)
    c = od.Context(cuda_device, 10, 10, 1, 1)
    yield c
    c.close()


def padded(x, fill=float("nan")):
    """The same rows, 16-byte strides; what lies behind a row is NaN."""
    per = 16 // x.element_size()
    store = torch.full((*x.shape[:-1], (x.shape[-1] // per + 2) * per), fill, dtype=x.dtype, device=x.device)
    store[..., :x.shape[-1]] = x
    return store[..., :x.shape[-1]]


def layer(V, H, G, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (V, H // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.rand(V, H // G, generator=g, device="cuda") + 0.1) * torch.where(torch.rand(V, H // G, generator=g, device="cuda") < 0.1, -1, 1)
    return codes, scales.to(BF16)


def weights(codes, scales):
    V, H = codes.shape[0], codes.shape[1] * 2
    w = torch.empty(V, H, dtype=torch.float64, device="cuda")
    w[:, 0::2], w[:, 1::2] = (codes % 16).double() - 8, (codes // 16).double() - 8
    return w * scales.double().repeat_interleave(H // scales.shape[1], 1)


def same(got, want, tol):
    got = got.double()
    tol = tol + HALF[F32] * want.abs()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}: {got[bad][:4].tolist()} for {want[bad][:4].tolist()}, tolerance {tol[bad][:4].tolist()}"


def magnitudes(codes, scales):
    """(u + 8) |s| of every weight."""
    return weights(codes, torch.ones_like(scales)).add_(16) * scales.double().abs().repeat_interleave(2 * codes.shape[1] // scales.shape[1], 1)


def check_logits(got, x, w, G, size_of):
    want, size = x.double() @ w.T, x.double().abs() @ size_of.T
    tol = size * (G / 16 * 3 * 2.0 ** -22 + (G / 8 + 2 + w.shape[1] / G + 4) * 2.0 ** -24)
    same(got, want, tol + HALF[got.dtype] * (want.abs() + tol))


def check_grad(got, dy, w, size_of):
    want, size = dy.double() @ w, dy.double().abs() @ size_of
    tol = size * (math.ceil(w.shape[0] / 16) * 3 * 2.0 ** -22 + 64 * 2.0 ** -24)
    same(got, want, tol + HALF[got.dtype] * (want.abs() + tol))


# tokens, vocabulary, hidden size, group
SIZES = [(1, 1, 32, 32), (2, 3, 64, 64), (1, 16, 128, 128), (7, 17, 96, 32), (8, 31, 1056, 32), (9, 100, 320, 64), (1, 1000, 768, 128),
         (16, 515, 4096, 128), (17, 2000, 1152, 64), (33, 333, 640, 32), (64, 1025, 512, 128), (5, 4099, 2048, 64), (3, 40, 16384, 128),
         (1, 9, 65536, 64), (12, 20011, 256, 32)]
TYPES = [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)]


@pytest.mark.parametrize("given,made", TYPES)
@pytest.mark.parametrize("N,V,H,G", SIZES)
def test_logits(ctx, N, V, H, G, given, made):
    codes, scales = layer(V, H, G, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = padded(torch.randn(N, H, generator=g, device="cuda").to(given))
    per = 16 // torch.empty(0, dtype=made).element_size()
    store = torch.full((N + 1, (V // per + 2) * per), 55.0, dtype=made, device="cuda")
    out = od.od_q4_logits(ctx, x, codes, scales, out=store[:N, :V])
    check_logits(out, x, weights(codes, scales), G, magnitudes(codes, scales))
    assert (store[N] == 55).all() and (store[:, V:] == 55).all()
    assert torch.equal(out, od.od_q4_logits(ctx, x, codes, scales, dtype=made))      # the same in every run


@pytest.mark.parametrize("given,made", TYPES)
@pytest.mark.parametrize("N,V,H,G", SIZES)
def test_gradient(ctx, N, V, H, G, given, made):
    codes, scales = layer(V, H, G, 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    dy = padded(torch.randn(N, V, generator=g, device="cuda").to(given))
    store = torch.full((N + 1, H + 32), 55.0, dtype=made, device="cuda")
    out = od.od_q4_logits_grad(ctx, dy, codes, scales, out=store[:N, :H])
    check_grad(out, dy, weights(codes, scales), magnitudes(codes, scales))
    assert (store[N] == 55).all() and (store[:, H:] == 55).all()
    assert torch.equal(out, od.od_q4_logits_grad(ctx, dy, codes, scales, dtype=made))


# positions: about what one launch takes, and of several; short layers and ones that a second kernel joins
@pytest.mark.parametrize("given,made", TYPES)
@pytest.mark.parametrize("N,V,H,G", [(23, 40, 128, 32), (24, 3001, 1152, 64), (25, 517, 640, 32), (31, 33, 2048, 128), (32, 20003, 256, 32),
                                     (40, 4100, 1024, 128), (41, 700, 96, 32), (56, 1000, 2048, 64)])
def test_gradient_of_more_positions(ctx, N, V, H, G, given, made):
    test_gradient(ctx, N, V, H, G, given, made)


def test_every_code_and_column(ctx):
    """Unit vectors read single weights: every code at every place of a word, each group's own scale."""
    V, H, G = 16, 256, 64
    u = (torch.arange(V, device="cuda")[:, None] + 5 * torch.arange(H, device="cuda")[None]) % 16
    codes = (u[:, 0::2] | u[:, 1::2] << 4).to(torch.uint8)
    scales = (2.0 ** (torch.arange(V, device="cuda")[:, None] - 2.0 * torch.arange(H // G, device="cuda")[None])).to(BF16)
    w = weights(codes, scales)
    for dtype in (BF16, F32):
        assert torch.equal(od.od_q4_logits(ctx, torch.eye(H, device="cuda").to(dtype), codes, scales).double(), w.T)
        assert torch.equal(od.od_q4_logits_grad(ctx, torch.eye(V, device="cuda").to(dtype), codes, scales).double(), w)


def test_fp32_inputs_keep_their_digits(ctx):
    """Inputs that differ in their last bits only: what is left of them after they cancel."""
    V, H, G = 40, 64, 32
    codes = torch.full((V, H // 2), 0x97, dtype=torch.uint8, device="cuda")          # -1 in even columns, +1 in odd ones
    scales = torch.ones(V, H // G, dtype=BF16, device="cuda")
    x = torch.zeros(1, H, device="cuda")
    x[0, 6], x[0, 7] = 1.0 + 2.0 ** -23, 1.0 + 3 * 2.0 ** -23
    assert (od.od_q4_logits(ctx, x, codes, scales) == 2.0 ** -22).all()
    codes[0::2] = 0x79
    dy = padded(torch.zeros(1, V, device="cuda"))
    dy[0, 4], dy[0, 5] = 1.0 + 2.0 ** -23, 1.0 + 3 * 2.0 ** -23
    got = od.od_q4_logits_grad(ctx, dy, codes, scales)
    assert (got[0, 0::2] == -2.0 ** -22).all() and (got[0, 1::2] == 2.0 ** -22).all()


def test_a_gradient_of_one_sign(ctx):
    """A softmax but for one entry through a long layer, one scale everywhere: the sums' errors are those of random signs. With
    steps of fp32 (2^-24) that are off by half of one at most and to either side, 16 parts of some thousand rows stay within
    2^-19 of the root of the sum of squares and of the large entry's weights."""
    N, V, H, G = 8, 30000, 256, 64
    codes, scales = layer(V, H, G, 30)
    scales.fill_(1.0)
    g = torch.Generator(device="cuda").manual_seed(31)
    dy = torch.softmax(torch.randn(N, V, generator=g, device="cuda") * 3, 1)
    dy[torch.arange(N), torch.randint(0, V, (N,), generator=g, device="cuda")] -= 1.0
    w = weights(codes, scales)
    want = dy.double() @ w
    got = od.od_q4_logits_grad(ctx, padded(dy), codes, scales).double()
    assert float((got - want).norm() / want.norm()) <= 2.0 ** -19


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_inputs_at_the_limits(ctx, dtype):
    """Infinities and NaN reach the results that the formula has them in, and no others; the largest and smallest finite values stay finite."""
    N, V, H, G = 9, 50, 128, 32
    codes, scales = layer(V, H, G, 5)
    codes[:, 3] = 0x99                                      # columns 6 and 7: +1 everywhere
    w = weights(codes, scales)
    x = torch.randn(N, H, device="cuda").to(dtype)
    x[1, 6], x[2, 6], x[3, 6] = math.inf, -math.inf, float("nan")
    y = od.od_q4_logits(ctx, x, codes, scales)
    sign = torch.sign(w[:, 6])
    assert torch.equal(y[1], (sign * math.inf).float()) and torch.equal(y[2], (-sign * math.inf).float()) and torch.isnan(y[3]).all()
    keep = [0, 4, 5, 6, 7, 8]
    check_logits(y[keep], x[keep], w, G, magnitudes(codes, scales))
    dy = padded(torch.randn(N, V, device="cuda").to(dtype))
    codes[4] = 0x99
    w = weights(codes, scales)
    dy[1, 4], dy[2, 4] = math.inf, float("nan")
    dx = od.od_q4_logits_grad(ctx, dy, codes, scales)
    assert torch.equal(dx[1], (torch.sign(w[4]) * math.inf).float()) and torch.isnan(dx[2]).all()
    keep = [0] + list(range(3, N))
    check_grad(dx[keep], dy[keep], w, magnitudes(codes, scales))
    # the type's largest value, and tiny ones, through weights of a half
    codes.fill_(0x88); codes[:, 0] = 0x89; scales.fill_(0.5)
    x = torch.zeros(2, H, device="cuda", dtype=dtype)
    x[0, 0], x[1, 0] = torch.finfo(dtype).max, 2.0 ** -126
    # (a product x u with u = 9, a beginning of -8 x: the six instructions of its group in fp32 meet 17 x at most)
    check_logits(od.od_q4_logits(ctx, x, codes, scales), x, weights(codes, scales), G, magnitudes(codes, scales))
    dy = padded(torch.zeros(2, V, device="cuda", dtype=dtype))
    dy[0, 3], dy[1, 3] = torch.finfo(dtype).max, 2.0 ** -110
    check_grad(od.od_q4_logits_grad(ctx, dy, codes, scales), dy, weights(codes, scales), magnitudes(codes, scales))


def test_the_gradient_is_the_transpose(ctx):
    """<y, dy> = <x, dx>: the two products use the same weights."""
    N, V, H, G = 6, 700, 384, 64
    codes, scales = layer(V, H, G, 6)
    x, dy = torch.randn(N, H, device="cuda"), padded(torch.randn(N, V, device="cuda"))
    a = (od.od_q4_logits(ctx, x, codes, scales).double() * dy.double()).sum()
    b = (od.od_q4_logits_grad(ctx, dy, codes, scales).double() * x.double()).sum()
    w = weights(codes, scales)
    size = float((x.double().abs() @ magnitudes(codes, scales).T * dy.double().abs()).sum())
    assert abs(float(a - b)) <= size * (2.0 ** -17 + math.ceil(V / 16) * 3 * 2.0 ** -22)


def test_codes_past_32_bits(ctx):
    """More than 2^32 weights, a token's worth of them checked."""
    V, H, G = 70000, 65536, 128
    codes = torch.randint(0, 256, (V, H // 2), device="cuda", dtype=torch.uint8)
    scales = torch.ones(V, H // G, dtype=BF16, device="cuda") / 16
    x = torch.randn(1, H, device="cuda").to(BF16)
    y = od.od_q4_logits(ctx, x, codes, scales)
    rows = torch.tensor([0, 1, 32767, 32768, 65535, 65536, 69998, V - 1], device="cuda")
    check_logits(y[:, rows], x, weights(codes[rows], scales[rows]), G, magnitudes(codes[rows], scales[rows]))
    dy = padded(torch.zeros(1, V, device="cuda"))
    dy[0, rows] = torch.randn(len(rows), device="cuda")
    check_grad(od.od_q4_logits_grad(ctx, dy, codes, scales), dy[:, rows], weights(codes[rows], scales[rows]), magnitudes(codes[rows], scales[rows]))


def test_batches_of_rows_captured_and_replayed_on_another_stream(ctx):
    B, K, V, H, G = 3, 4, 1500, 512, 128
    codes, scales = layer(V, H, G, 7)
    w = weights(codes, scales)
    x = torch.randn(B, K, H, device="cuda").to(BF16)
    logits = padded(torch.zeros(B, K, V, device="cuda"))
    back = torch.empty(B, K, H, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        od.od_q4_logits(ctx, x, codes, scales, out=logits)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            od.od_q4_logits(ctx, x, codes, scales, out=logits)
            od.od_q4_logits_grad(ctx, logits, codes, scales, out=back)
        x.copy_(torch.randn(B, K, H, device="cuda"))
        graph.replay()
    torch.cuda.synchronize()
    check_logits(logits.reshape(-1, V), x.view(-1, H), w, G, magnitudes(codes, scales))
    check_grad(back.view(-1, H), logits.reshape(-1, V), w, magnitudes(codes, scales))


def test_a_training_step_of_the_drafter(ctx):
    """Hidden states -> logits -> scores -> the gradient of a loss on them -> the hidden states' gradient, against autograd in 64 bits."""
    B, K, V, H, G, n = 3, 5, 3001, 256, 64, 4
    codes, scales = layer(V, H, G, 8)
    scales = (scales.float() / 64).to(BF16)
    w = weights(codes, scales)
    hidden = torch.randn(B, K, H, device="cuda").to(BF16)
    T = torch.tensor([1.0, 0.7, 0.5], device="cuda")
    ids = torch.randint(0, V, (B, K), device="cuda", dtype=torch.int32)
    n_rows = torch.tensor([5, 3, 4], dtype=torch.int32, device="cuda")
    live = torch.arange(K, device="cuda")[None] < n_rows[:, None]
    logits = od.od_q4_logits(ctx, hidden, codes, scales)
    lp = od.od_token_logprobs(ctx, logits, ids, T, n_rows, n)
    a, b = torch.randn(B, K, device="cuda"), torch.randn(B, K, device="cuda")
    c = torch.randn(B, K, n, device="cuda")
    g_logits = od.od_token_logprobs_grad(ctx, logits, ids, lp, a, b, c, T, n_rows)
    got = od.od_q4_logits_grad(ctx, g_logits, codes, scales)
    h = hidden.double().requires_grad_()
    ref = torch.log_softmax(h @ w.T / T.double()[:, None, None], 2)
    top = torch.gather(ref, 2, torch.where(live[:, :, None], lp.top_ids, 0).long())
    assert torch.equal(lp.top_ids[live].long(), torch.topk(ref, n, dim=2).indices[live])
    loss = (a * torch.gather(ref, 2, ids.long()[:, :, None]).squeeze(2) - b * (ref.exp() * ref).sum(2) + (c * top).sum(2))[live].sum()
    loss.backward()
    # the logits' errors (group sums of |x w|) through a softmax, then the tolerances of the two gradients
    size = float((hidden.double().abs() @ magnitudes(codes, scales).T).max())
    spread = (a.abs() + 16 * b.abs() + c.abs().sum(2)).double()[:, :, None] * w.abs().max() * 2 / T.double()[:, None, None]
    tol = spread * (size * 2.0 ** -18 * 4 + 2.0 ** -14)
    assert ((got.double() - h.grad).abs() <= tol)[live].all()
    assert not got[~live].any()


def test_refusals(ctx):
    codes, scales = layer(100, 128, 32, 9)
    x = torch.randn(2, 128, device="cuda")
    od.od_q4_logits(ctx, x, codes, scales)
    with pytest.raises(TypeError):
        od.od_q4_logits(ctx, x.half(), codes, scales)
    with pytest.raises(TypeError):
        od.od_q4_logits(ctx, x, codes.int(), scales)
    with pytest.raises(TypeError):
        od.od_q4_logits(ctx, x, codes, scales.float())
    with pytest.raises(ValueError):
        od.od_q4_logits(ctx, x[:, :64], codes, scales)
    with pytest.raises(ValueError):
        od.od_q4_logits(ctx, x, codes, scales[:50])
    with pytest.raises(ValueError):
        od.od_q4_logits(ctx, x, codes[:, ::2], scales)
    with pytest.raises(ValueError):
        od.od_q4_logits(ctx, x, codes, scales, out=torch.empty(3, 100, device="cuda"))
    with pytest.raises(ValueError):
        od.od_q4_logits(ctx, x.cpu(), codes, scales)
    with pytest.raises(ValueError):                         # rows that are not equally far apart
        od.od_q4_logits(ctx, torch.zeros(2, 3, 128, device="cuda")[:, :2], codes, scales)
    with pytest.raises(od.OdError) as e:
        od.od_q4_logits(ctx, x, codes, torch.zeros(100, 128 // 16, dtype=BF16, device="cuda"))
    assert e.value.status == od.OD_ERR_UNSUPPORTED
    with pytest.raises(od.OdError) as e:
        od.od_q4_logits(ctx, x, torch.zeros(100 * 64 + 1, dtype=torch.uint8, device="cuda")[1:].view(100, 64), scales)
    assert e.value.status == od.OD_ERR_ALIGNMENT
    with pytest.raises(od.OdError) as e:
        od.od_q4_logits(ctx, x, codes, scales, out=torch.empty(2, 101, device="cuda")[:, :100])
    assert e.value.status == od.OD_ERR_ALIGNMENT
    assert od.od_q4_logits(ctx, x[:0], codes, scales).shape == (0, 100)
    assert od.od_q4_logits_grad(ctx, torch.zeros(0, 100, device="cuda"), codes, scales).shape == (0, 128)


@pytest.mark.parametrize("call", [od.od_q4_logits, od.od_q4_logits_grad])
@pytest.mark.parametrize("given", [False, True])
def test_refuses_weights_of_other_dimensions(ctx, call, given):
    codes, scales = layer(128, 128, 32, 9)
    x = torch.randn(2, 128, device="cuda")
    out = torch.empty(2, 128, device="cuda") if given else None
    for c, s in [(codes.view(-1), scales), (codes[None], scales), (codes, scales.view(-1)), (codes, scales[None])]:
        with pytest.raises(ValueError):
            call(ctx, x, c, s, out=out)


def test_scales_far_from_one(ctx):
    """Scales that cannot be scaled up with the rest, and tiny ones, next to usual ones: groups of either kind in both directions."""
    N, V, H, G = 9, 70, 256, 64
    codes, scales = layer(V, H, G, 20)
    power = torch.tensor([0.0, 90.0, -90.0, 1.0], device="cuda")
    scales = (scales.double() * 2.0 ** power[None, :]).to(BF16)
    scales[5, 0], scales[6, 1] = 2.0 ** 70, 0.0
    x = torch.randn(N, H, device="cuda")
    x[:, G:2 * G] *= 2.0 ** -80
    x[3] = 0.0
    for dtype in (BF16, F32):
        xd = x.to(dtype)
        check_logits(od.od_q4_logits(ctx, xd, codes, scales), xd, weights(codes, scales), G, magnitudes(codes, scales))
    dy = torch.randn(N, V, device="cuda") * 2.0 ** -20
    dy[2] = 0.0
    for dtype in (BF16, F32):
        d = padded(dy.to(dtype))
        check_grad(od.od_q4_logits_grad(ctx, d, codes, scales), d, weights(codes, scales), magnitudes(codes, scales))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tokens_of_all_sizes_in_one_call(ctx, dtype):
    """Tokens of usual size, tiny, huge, all zeros and not finite beside one another."""
    N, V, H, G = 16, 100, 512, 128
    codes, scales = layer(V, H, G, 21)
    g = torch.Generator(device="cuda").manual_seed(22)
    x = torch.randn(N, H, generator=g, device="cuda", dtype=torch.float64)
    x *= 2.0 ** torch.tensor([0, -100, 90, 0, 59, 60, -30, -31, -126, 1, 20, -20, 0, 0, 3, -3.0], device="cuda", dtype=torch.float64)[:, None]
    x[3] = 0.0
    x = x.to(dtype)
    x[12, 7] = math.inf
    y = od.od_q4_logits(ctx, x, codes, scales)
    keep = [n for n in range(N) if n != 12]
    w, size_of = weights(codes, scales), magnitudes(codes, scales)
    check_logits(y[[n for n in keep if n != 8]], x[[n for n in keep if n != 8]], w, G, size_of)
    # (the least one's results are of the size of fp32's smallest numbers, 2^-149 apart)
    want = x[8].double() @ w.T
    assert ((y[8].double() - want).abs() <= x[8].double().abs() @ size_of.T * 2.0 ** -17 + 2.0 ** -148).all()
    assert not torch.isfinite(y[12][w[:, 7] != 0]).any()
    assert torch.equal(od.od_q4_logits(ctx, x[:1], codes, scales), od.od_q4_logits(ctx, x[:2], codes, scales)[:1])


def test_many_tokens(ctx):
    N, V, H, G = 131, 300, 384, 128
    codes, scales = layer(V, H, G, 23)
    w, size_of = weights(codes, scales), magnitudes(codes, scales)
    x, dy = torch.randn(N, H, device="cuda").to(BF16), padded(torch.randn(N, V, device="cuda").to(BF16))
    check_logits(od.od_q4_logits(ctx, x, codes, scales), x, w, G, size_of)
    check_grad(od.od_q4_logits_grad(ctx, dy, codes, scales), dy, w, size_of)


def test_two_streams_at_once(ctx):
    """od_q4_logits has no scratch: calls on one context need no order."""
    V, H, G = 20000, 1024, 64
    codes, scales = layer(V, H, G, 24)
    xs = [torch.randn(n, H, device="cuda").to(BF16) for n in (3, 20)]
    want = [od.od_q4_logits(ctx, x, codes, scales) for x in xs]
    out = [torch.zeros_like(y) for y in want]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, y, s in zip(xs, out, streams):
            with torch.cuda.stream(s):
                od.od_q4_logits(ctx, x, codes, scales, out=y)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_with_and_without_the_extension(ctx, monkeypatch):
    codes, scales = layer(100, 128, 32, 25)
    x, dy = torch.randn(2, 3, 128, device="cuda"), padded(torch.randn(2, 3, 100, device="cuda"))
    y, dx = torch.empty(2, 3, 100, device="cuda"), torch.empty(2, 3, 128, device="cuda")
    a = od.od_q4_logits(ctx, x, codes, scales, out=y).clone(), od.od_q4_logits_grad(ctx, dy, codes, scales, out=dx).clone()
    monkeypatch.setattr(od, "_native", od._InPython())
    b = od.od_q4_logits(ctx, x, codes, scales, out=y), od.od_q4_logits_grad(ctx, dy, codes, scales, out=dx)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_the_distillation_gradient_back_to_the_hidden_states(ctx):
    """A verified batch's distillation loss, its gradient and the drafter's 4-bit layer: d loss / d hidden against 64 bits."""
    from paper_2507_02659_b200 import synth
    import parity
    V_q, H, G = 1200, 256, 64
    w = synth.Workload("q4distill", B=4, steps=1, k_max=4, k_min=1, v_q=V_q, v_p=5003, logit_dtype="bf16", map_kind="random",
                       mapped_frac=0.7, cache_entries=100, hit_prob=0.3, logit_kind="corr", rho=0.95, temperatures=(1.0, 0.5),
                       per_seq_seed=True, gen_seed=0x5C1, unmapped_shift=2.0, sigma=2.0)
    st = synth.make_static(w)
    c = parity.make_context(w, st, "cuda:0")
    s = synth.make_step(w, st, 0, device="cuda:0")
    logits = parity.pad_rows(s.logits)
    mp = od.od_map_proposals(c, s.draft_ids, s.draft_len, s.q_sel)
    vo = od.od_verify(c, logits, mp, s.temperature, s.seed, 0)
    _, grad = od.od_distill_loss(c, s.q_rows, s.draft_ids, mp, logits, vo, s.temperature, 0.2)
    codes, scales = layer(V_q, H, G, 26)
    got = od.od_q4_logits_grad(c, grad, codes, scales)
    check_grad(got.view(-1, H), grad.view(-1, V_q), weights(codes, scales), magnitudes(codes, scales))
    c.close()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["one sign", "a mean", "equal"])
@pytest.mark.parametrize("N,V,H,G", [(8, 4096, 4096, 128), (5, 1000, 768, 64), (12, 700, 2048, 32), (3, 500, 8192, 128)])
def test_inputs_of_one_sign(ctx, N, V, H, G, kind, dtype):
    """Sums of inputs that do not cancel are as good as sums of fp32 steps to either side. Steps of bf16 inputs meet up to 8 sum |x| of a
    group, 16 times its sum's root mean square for 128 columns, half of it on the way: eight steps of 2^-24 of that at most, evenly spread, are
    8e-7 of it, and errors of different groups do not add up more than the groups do. fp32 inputs' steps meet the sums alone: cut
    by 2^-23 each and all to one side they are 2^-20 of them. Both are below 2^-19 with the sums over groups."""
    _, scales = layer(V, H, G, 32)
    scales = scales.abs()
    g = torch.Generator(device="cuda").manual_seed(33)
    u = torch.round(8 + 2.3 * torch.randn(V, H, generator=g, device="cuda")).clamp(0, 15).to(torch.uint8)     # (of mean zero less 8)
    codes = u[:, 0::2] | u[:, 1::2] << 4
    x = torch.randn(N, H, generator=g, device="cuda")
    x = {"one sign": x.abs(), "a mean": x + 3, "equal": torch.full_like(x, 1.1)}[kind].to(dtype)
    want = x.double() @ weights(codes, scales).T
    got = od.od_q4_logits(ctx, x, codes, scales).double()
    assert float((got - want).norm() / want.norm()) <= 2.0 ** -19


def test_the_first_calls_of_a_process_are_captured():
    """What kernels need is set at their first launch: into a graph too."""
    import os
    import subprocess
    import sys
    program = """
import torch
from paper_2507_02659_b200 import binding as od
ctx = od.Context("cuda:0", 10, 10, 1, 1)
g = torch.Generator(device="cuda").manual_seed(1)
V, H = 20003, 1024
codes = torch.randint(0, 256, (V, H // 2), generator=g, device="cuda", dtype=torch.uint8)
scales = torch.rand(V, H // 64, generator=g, device="cuda").bfloat16()
for n, dtype in ((7, torch.bfloat16), (20, torch.float32), (40, torch.bfloat16)):
    x = torch.randn(n, H, generator=g, device="cuda").to(dtype)
    y, dx = torch.zeros(n, V // 4 * 4 + 4, device="cuda")[:, :V], torch.zeros(n, H, device="cuda", dtype=dtype)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        od.od_q4_logits(ctx, x, codes, scales, out=y)
        od.od_q4_logits_grad(ctx, y, codes, scales, out=dx)
    graph.replay()
    want = od.od_q4_logits(ctx, x, codes, scales)
    back = od.od_q4_logits_grad(ctx, want, codes, scales, dtype=dtype)
    assert want.any() and back.any() and torch.equal(y, want) and torch.equal(dx, back), n
ctx.close()
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", program], check=True, cwd=root, timeout=300)


@pytest.mark.parametrize("given,made", TYPES)
@pytest.mark.parametrize("N", [1, 8, 16, 24, 32, 40])
@pytest.mark.parametrize("V,H,G", [(20011, 256, 32), (20003, 2048, 128), (30001, 1152, 64)])
def test_gradients_through_long_layers(ctx, V, H, G, N, given, made):
    """Errors of the whole, where the bound for single results lets some hundred rows go missing. A warp has at most every eighth 32
    rows of its block, and blocks share the rows of these layers by 18 and more, up to 14 stages of 2 x 3 instructions: as fp32
    steps to either side (2^-24 of the sum) they are off by 2^-20 of it and so is what joins 148 parts: 2^-19 of the norm. Cut by 2^-23
    each and all to one side they are 2^-16 of the results' root mean square at a single one that is written as bf16."""
    codes, scales = layer(V, H, G, 34)
    w = weights(codes, scales)
    g = torch.Generator(device="cuda").manual_seed(35)
    dy = padded(torch.randn(N, V, generator=g, device="cuda").to(given))
    want = dy.double() @ w
    got = od.od_q4_logits_grad(ctx, dy, codes, scales, dtype=made).double()
    if made == F32:
        assert float((got - want).norm() / want.norm()) <= 2.0 ** -19
    else:
        same(got, want, HALF[BF16] * want.abs() + 2.0 ** -16 * want.square().mean().sqrt())
    # rows at the ends of the layer and of stages alone: none of them is left out, nor counted twice
    rows = torch.tensor([0, 15, 16, 31, 32, 255, 256, V // 64 * 32 - 1, V // 64 * 32, V // 32 * 32 - 33, V // 32 * 32 - 1, V // 32 * 32, V - 1], device="cuda")
    for r in (rows, rows[-1:], rows[-2:-1]):
        few = torch.zeros_like(dy)
        few[:, r] = dy[:, r]
        check_grad(od.od_q4_logits_grad(ctx, padded(few), codes, scales, dtype=made), few[:, r], w[r], magnitudes(codes[r], scales[r]))
