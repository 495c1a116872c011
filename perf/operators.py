"""The scores of tokens and a drafter's 4-bit output layer, each with its gradient, as timed cases.

Four operators: the log probability of a given token, the entropy and the likeliest tokens of
each logit row (`logprobs`) and the gradient of all three (`logprobs_grad`); the logits of a few
tokens from an output layer whose weights are 4-bit codes with a scale for every group of columns
(`q4`) and the way of a logit gradient back through it (`q4_grad`). Where `own` is false they are
computed in elementary torch operations in 32 bits, where it is true by the library.

`listed()` holds the cases that are always timed, `draw()` gives more of the same ranges.
"""
import math

import torch

own = False

SIGMA = 3.0             # spread of a row's logits
HEAD = 256              # ids of a row that stand out, Zipf-ranked
MASKED_SHARE = 0.3      # ids that a constrained row leaves out (-inf)

DEFAULTS = dict(op="logprobs", B=1, R=1, V=32000, dtype="bf16", ragged=False, top=0, masked=False, entropy=True,
                N=1, H=1024, G=128, out="f32")


def _case(name, **kw):
    return dict(DEFAULTS, name=name, **kw)


def listed():
    return [
        # one user, the token that the drafter has just proposed, with five alternatives: all latency
        _case("lp_one_32k_f32", B=1, R=1, V=32000, dtype="f32", top=5),
        # a server's answer for two dozen users: every verified position with twenty alternatives
        _case("lp_24x7_128k_top20", B=24, R=7, V=128256, ragged=True, top=20),
        # rows that are multiples of nothing, in fp32, of a constrained vocabulary
        _case("lp_19x6_odd_f32", B=19, R=6, V=100277, dtype="f32", ragged=True, top=3, masked=True),
        # the largest batch scored whole, only the likeliest token besides
        _case("lp_512x9_152k", B=512, R=9, V=152064, top=1),
        # training on one user's proposals, small vocabulary: the smallest gradient
        _case("lpg_1x4_32k_f32", op="logprobs_grad", B=1, R=4, V=32000, dtype="f32"),
        # training on a verified batch: likelihood and entropy
        _case("lpg_64x7_128k", op="logprobs_grad", B=64, R=7, V=128256, ragged=True),
        # the same for a few users, fp32 logits, the alternatives' log probabilities in the loss too
        _case("lpg_5x11_152k_f32_top8", op="logprobs_grad", B=5, R=11, V=152064, dtype="f32", top=8),
        # one draft token on the device: the smallest output layer
        _case("q4_1_32k_768", op="q4", N=1, V=32000, H=768, G=32),
        # eight users' draft tokens through the widest layer of the largest vocabulary
        _case("q4_8_128k_4096", op="q4", N=8, V=128256, H=4096, G=128, out="bf16"),
        # sizes that are multiples of nothing, hidden states in fp32
        _case("q4_5_odd_f32", op="q4", N=5, V=31991, H=1056, G=32, dtype="f32"),
        # the distillation gradient of one user's six positions back to the hidden states
        _case("q4g_6_32k_768_f32", op="q4_grad", N=6, V=32000, H=768, G=64, dtype="f32"),
        # two dozen positions through a wide layer
        _case("q4g_24_128k_2048", op="q4_grad", N=24, V=128256, H=2048, G=128, out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(DEFAULTS, op=rng.choice(["logprobs", "logprobs_grad", "q4", "q4_grad"]))
    c["V"] = rng.choice([32000, 128256, 152064]) if rng.random() < 0.4 else _log_int(rng, 8000, 152064)
    c["dtype"] = "bf16" if rng.random() < 0.6 else "f32"
    if c["op"] in ("logprobs", "logprobs_grad"):
        c["B"], c["R"] = _log_int(rng, 1, 512), rng.randint(1, 17)
        c["ragged"] = rng.random() < 0.5
        c["masked"] = rng.random() < 0.3
        c["top"] = rng.choice([0, 1, rng.randint(2, 20)])
        c["entropy"] = rng.random() < 0.8
        cap = 1.4e9 if c["op"] == "logprobs" else 4e8
        while c["B"] > 1 and work(c)["bytes"] > cap:
            c["B"] = c["B"] * 3 // 4
    else:
        c["N"] = _log_int(rng, 1, 64)
        c["G"] = rng.choice([32, 64, 128])
        c["H"] = c["G"] * max(1, _log_int(rng, 512, 4096) // c["G"])
        c["out"] = rng.choice(["bf16", "f32"])
        cap = 2.7e8 * 8 if c["op"] == "q4" else 1.4e8 * 24      # bytes of codes times tokens
        while c["N"] > 1 and c["N"] * c["V"] * c["H"] / 2 > cap:
            c["N"] = c["N"] * 3 // 4
    return c


def _esz(name):
    return 2 if name == "bf16" else 4


def _torch(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _row_counts(c):
    """Rows that count of each sequence's R."""
    return [1 + (7 * b + 3) % c["R"] if c["ragged"] else c["R"] for b in range(c["B"])]


def work(case):
    c = dict(DEFAULTS, **case)
    if c["op"] in ("q4", "q4_grad"):
        e = c["V"] * c["H"]
        hidden, logits = c["N"] * c["H"], c["N"] * c["V"]
        first, second = (hidden, logits) if c["op"] == "q4" else (logits, hidden)
        return {"bytes": e // 2 + e // c["G"] * 2 + first * _esz(c["dtype"]) + second * _esz(c["out"]),
                "flops": 2 * c["N"] * e}
    rows = sum(_row_counts(c))
    if c["op"] == "logprobs":
        return {"bytes": rows * (c["V"] * _esz(c["dtype"]) + 4 + 20 + 8 * c["top"]), "flops": 6 * rows * c["V"]}
    # rows that do not count have a gradient too: zeros
    return {"bytes": (rows + c["B"] * c["R"]) * c["V"] * _esz(c["dtype"]) + rows * (24 + 8 * c["top"]),
            "flops": 7 * rows * c["V"]}


# ---- inputs ------------------------------------------------------------------------------

def _rows(c, g):
    """Logits [B, R, V] with rows padded to 16 bytes, the given ids [B, R] (every 16th row has none)."""
    B, R, V = c["B"], c["R"], c["V"]
    dev, dtype = "cuda", _torch(c["dtype"])
    per = 16 // _esz(c["dtype"])
    store = torch.zeros(B, R, (V + per - 1) // per * per, dtype=dtype, device=dev)
    zipf = 12.0 - 1.1 * torch.log(torch.arange(1, HEAD + 1, device=dev, dtype=torch.float32))
    out_of = torch.rand(V, generator=g, device=dev) < MASKED_SHARE
    ids = torch.empty(B, R, dtype=torch.int32, device=dev)
    for lo in range(0, B, 64):
        hi = min(B, lo + 64)
        x = torch.randn(hi - lo, R, V, generator=g, device=dev) * SIGMA
        # (ids 31 apart are all different: V is at least 8000)
        head = (torch.randint(0, V, (hi - lo, R, 1), generator=g, device=dev) + 31 * torch.arange(HEAD, device=dev)) % V
        x.scatter_(2, head, x.gather(2, head) + zipf)
        if c["masked"]:
            x.masked_fill_(out_of, -math.inf)
        store[lo:hi, :, :V] = x.to(dtype)
        # the given token is mostly a likely one
        rank = (torch.rand(hi - lo, R, 1, generator=g, device=dev) ** 4 * HEAD).long().clamp(max=HEAD - 1)
        ids[lo:hi] = torch.gather(head, 2, rank).squeeze(2).int()
    ids.view(-1)[15::16] = -1
    return store[:, :, :V], ids


def _weights(c, g):
    """Codes uint8 [V, H / 2] (column 2i in the low half of byte i) and scales bf16 [V, H / G]."""
    V, H, G = c["V"], c["H"], c["G"]
    codes = torch.empty(V, H // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(V, H // G, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, V, 16384):
        hi = min(V, lo + 16384)
        w = torch.randn(hi - lo, H // G, G, generator=g, device="cuda") / math.sqrt(H)
        s = (w.abs().amax(2) / 7.0).to(torch.bfloat16)
        u = (torch.round(w / s.float()[:, :, None]) + 8.0).clamp(0, 15).to(torch.uint8).view(hi - lo, H)
        codes[lo:hi] = u[:, 0::2] | u[:, 1::2] << 4
        scales[lo:hi] = s
    return codes, scales


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = "cuda"
    s = {}
    if c["op"] in ("logprobs", "logprobs_grad"):
        B, R, n = c["B"], c["R"], c["top"]
        s["logits"], s["ids"] = _rows(c, g)
        s["temperature"] = torch.tensor([0.5, 0.7, 1.0], device=dev).repeat(-(-B // 3))[:B].contiguous()
        s["n_rows"] = torch.tensor(_row_counts(c), dtype=torch.int32, device=dev) if c["ragged"] else None
        if c["op"] == "logprobs_grad":
            s["g_logprob"] = torch.randn(B, R, generator=g, device=dev)
            s["g_entropy"] = torch.randn(B, R, generator=g, device=dev) * 0.1 if c["entropy"] else None
            s["g_top"] = torch.randn(B, R, n, generator=g, device=dev) if n else None
        return s
    s["codes"], s["scales"] = _weights(c, g)
    N, V, H = c["N"], c["V"], c["H"]
    if c["op"] == "q4":
        # normalised hidden states, a few columns far larger than the rest
        x = torch.randn(N, H, generator=g, device=dev)
        x[:, torch.randint(0, H, (4,), generator=g, device=dev)] *= 20.0
        s["hidden"] = x.to(_torch(c["dtype"]))
    else:
        # softmax minus the proposed token: a few large entries, many small ones
        per = 16 // _esz(c["dtype"])
        store = torch.zeros(N, (V + per - 1) // per * per, dtype=_torch(c["dtype"]), device=dev)
        z = torch.softmax(torch.randn(N, V, generator=g, device=dev) * SIGMA, 1)
        z[torch.arange(N, device=dev), torch.randint(0, V, (N,), generator=g, device=dev)] -= 1.0
        store[:, :V] = z.to(store.dtype)
        s["g_logits"] = store[:, :V]
    return s


def prepare(case, seed):
    c = dict(DEFAULTS, **case)
    s = dict(_inputs(c, seed), case=c)
    if c["op"] in ("logprobs", "logprobs_grad"):
        # what the forward pass leaves, and buffers for what it writes (rows that do not count stay as they are)
        B, R, n = c["B"], c["R"], c["top"]
        z = lambda *shape, dt=torch.float32: torch.zeros(*shape, dtype=dt, device="cuda")
        s["out"] = dict(logprob=z(B, R), entropy=z(B, R), row_max=z(B, R), row_sum=z(B, R),
                        top_ids=z(B, R, n, dt=torch.int32), top_logprobs=z(B, R, n), flags=z(B, R, dt=torch.int32))
        if c["op"] == "logprobs_grad":
            s["out"] = _plain_logprobs(s, s["out"])
            s["grad"] = torch.empty_strided(s["logits"].shape, s["logits"].stride(), dtype=s["logits"].dtype, device="cuda")
    else:
        N, V, H = c["N"], c["V"], c["H"]
        per = 16 // _esz(c["out"])
        s["y"] = (torch.empty(N, (V + per - 1) // per * per, dtype=_torch(c["out"]), device="cuda")[:, :V]
                  if c["op"] == "q4" else torch.empty(N, H, dtype=_torch(c["out"]), device="cuda"))
    if own:
        from paper_2507_02659_b200 import binding as od
        s["ctx"] = od.Context("cuda", c["V"], c["V"], 1, 1)
        if "out" in s:
            s["out"] = od.LogprobOut(**s["out"])
    return s


# ---- one pass ----------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "logprobs":
        return _plain_logprobs(s, s["out"])
    if c["op"] == "logprobs_grad":
        return _plain_logprobs_grad(s)
    w = _plain_weights(c, s["codes"], s["scales"])
    if c["op"] == "q4":
        return (s["hidden"].float() @ w.T).to(_torch(c["out"]))
    return (s["g_logits"].float() @ w).to(_torch(c["out"]))


def _run_own(s, c):
    from paper_2507_02659_b200 import binding as od
    if c["op"] == "logprobs":
        return vars(od.od_token_logprobs(s["ctx"], s["logits"], s["ids"], temperature=s["temperature"],
                                         n_rows=s["n_rows"], n_top=c["top"], out=s["out"]))
    if c["op"] == "logprobs_grad":
        return od.od_token_logprobs_grad(s["ctx"], s["logits"], s["ids"], s["out"], s["g_logprob"],
                                         g_entropy=s["g_entropy"], g_top=s["g_top"], temperature=s["temperature"],
                                         n_rows=s["n_rows"], grad=s["grad"])
    if c["op"] == "q4":
        return od.od_q4_logits(s["ctx"], s["hidden"], s["codes"], s["scales"], out=s["y"])
    return od.od_q4_logits_grad(s["ctx"], s["g_logits"], s["codes"], s["scales"], out=s["y"])


def _live(s, B, R):
    r = torch.arange(R, device="cuda")[None, :]
    return (r < s["n_rows"][:, None]) if s["n_rows"] is not None else torch.ones(B, R, dtype=torch.bool, device="cuda")


def _chunks(B, R, V):
    """Sequences at a time: about 2^26 elements."""
    n = max(1, (1 << 26) // (R * V))
    return [(lo, min(B, lo + n)) for lo in range(0, B, n)]


def _plain_logprobs(s, out):
    """Rows without a finite positive sum do not occur here; logits may be -inf."""
    logits, ids = s["logits"], s["ids"]
    B, R, V = logits.shape
    n = out["top_ids"].shape[2]
    live = _live(s, B, R)
    got = {k: torch.empty_like(t) for k, t in out.items()}
    for lo, hi in _chunks(B, R, V):
        x = logits[lo:hi].float()
        T = s["temperature"][lo:hi, None, None]
        M = x.max(2, keepdim=True).values
        d = (x - M) / T
        e = torch.exp(d)
        S = e.sum(2, keepdim=True)
        ln = torch.log(S)
        got["row_max"][lo:hi], got["row_sum"][lo:hi] = M.squeeze(2), S.squeeze(2)
        got["entropy"][lo:hi] = (ln - (e * torch.where(e > 0, d, 0.0)).sum(2, keepdim=True) / S).squeeze(2)
        lp = d - ln
        t = ids[lo:hi].long()
        at = torch.gather(lp, 2, t.clamp(min=0)[:, :, None]).squeeze(2)
        got["logprob"][lo:hi] = torch.where(t >= 0, at, 0.0)
        if n:
            # by value, then by the lower id: one whole number that orders so
            bits = (x + 0.0).view(torch.int32).long()
            key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * (1 << 32) - torch.arange(V, device="cuda")
            top = torch.topk(key, min(n, V), dim=2).indices
            value = torch.gather(lp, 2, top)
            got["top_ids"][lo:hi] = torch.where(value > -math.inf, top, -1).int()
            got["top_logprobs"][lo:hi] = value
    got["flags"].zero_()
    return {k: torch.where(live.view(B, R, *[1] * (t.dim() - 2)), got[k], t) for k, t in out.items()}


def _plain_logprobs_grad(s):
    logits, ids, out = s["logits"], s["ids"], s["out"]
    B, R, V = logits.shape
    live = _live(s, B, R)
    grad = torch.empty_like(s["grad"])
    for lo, hi in _chunks(B, R, V):
        T = s["temperature"][lo:hi, None, None]
        d = (logits[lo:hi].float() - out["row_max"][lo:hi, :, None]) / T
        S = out["row_sum"][lo:hi, :, None]
        p = torch.exp(d) / S
        t = ids[lo:hi].long()
        given = torch.where(t >= 0, s["g_logprob"][lo:hi], 0.0)
        total = given[:, :, None].clone()
        if s["g_top"] is not None:
            top = out["top_ids"][lo:hi].long()
            listed_ = torch.where(top >= 0, s["g_top"][lo:hi], 0.0)
            total += listed_.sum(2, keepdim=True)
        v = -p * total
        if s["g_entropy"] is not None:
            ln_p = torch.where(p > 0, d - torch.log(S), 0.0)
            v -= p * (ln_p + out["entropy"][lo:hi, :, None]) * s["g_entropy"][lo:hi, :, None]
        v.scatter_add_(2, t.clamp(min=0)[:, :, None], given[:, :, None])
        if s["g_top"] is not None:
            v.scatter_add_(2, top.clamp(min=0), listed_)
        grad[lo:hi] = torch.where(live[lo:hi, :, None], v / T, 0.0).to(grad.dtype)
    return grad


def _plain_weights(c, codes, scales):
    u = torch.stack((codes & 15, codes >> 4), 2).view(c["V"], c["H"] // c["G"], c["G"])
    return ((u.float() - 8.0) * scales.float()[:, :, None]).view(c["V"], c["H"])


# ---- the definitions in 64 bits -----------------------------------------------------------

def exact(case, seed):
    c = dict(DEFAULTS, **case)
    s = _inputs(c, seed)
    if c["op"] in ("q4", "q4_grad"):
        x = s["hidden" if c["op"] == "q4" else "g_logits"].double()
        y = x.new_empty(c["N"], c["V"]) if c["op"] == "q4" else x.new_zeros(c["N"], c["H"])
        for lo in range(0, c["V"], 8192):
            code = s["codes"][lo:lo + 8192].long()
            w = torch.empty(code.shape[0], c["H"], dtype=torch.float64, device="cuda")
            w[:, 0::2], w[:, 1::2] = (code % 16 - 8).double(), (code // 16 - 8).double()
            w *= torch.repeat_interleave(s["scales"][lo:lo + 8192].double(), c["G"], dim=1)
            if c["op"] == "q4":
                y[:, lo:lo + 8192] = x @ w.T
            else:
                y += x[:, lo:lo + 8192] @ w
        return y
    B, R, V, n = c["B"], c["R"], c["V"], c["top"]
    counts = _row_counts(c)
    f = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")
    out = dict(logprob=f(B, R), entropy=f(B, R), row_max=f(B, R), row_sum=f(B, R),
               top_ids=torch.zeros(B, R, n, dtype=torch.int64, device="cuda"), top_logprobs=f(B, R, n),
               flags=torch.zeros(B, R, dtype=torch.int64, device="cuda"))
    grad = f(B, R, V) if c["op"] == "logprobs_grad" else None
    for b in range(B):
        k = counts[b]
        x = s["logits"][b, :k].double() / s["temperature"][b].double()
        lp = torch.log_softmax(x, 1)
        p = torch.exp(lp)
        H = -torch.nan_to_num(p * lp, nan=0.0).sum(1)
        ids = s["ids"][b, :k].long()
        has = ids >= 0
        row = torch.arange(k, device="cuda")
        if grad is None or n:
            # a stable order keeps equal values by id; only the first of it is needed
            bound = torch.topk(x, min(n, V), dim=1).values[:, -1:] if n else x
            for r in range(k if n else 0):
                near = torch.nonzero((x[r] >= bound[r]) & (x[r] > -math.inf)).squeeze(1)
                first = near[torch.argsort(x[r, near], descending=True, stable=True)][:n]
                out["top_ids"][b, r] = -1
                out["top_logprobs"][b, r] = -math.inf
                out["top_ids"][b, r, :first.numel()] = first
                out["top_logprobs"][b, r, :first.numel()] = lp[r, first]
        if grad is None:
            out["logprob"][b, :k] = torch.where(has, lp[row, ids.clamp(min=0)], 0.0)
            out["entropy"][b, :k] = H
            out["row_max"][b, :k] = s["logits"][b, :k].double().max(1).values
            out["row_sum"][b, :k] = torch.exp(x - x.max(1, keepdim=True).values).sum(1)
            continue
        # d logprob_i / dx = (one at i) - p, d H / dx = -p (ln p + H), all over T
        g = torch.where(has, s["g_logprob"][b, :k].double(), 0.0)
        v = torch.zeros_like(x)
        v[row, ids.clamp(min=0)] += g
        if n:
            top = out["top_ids"][b, :k]
            gt = torch.where(top >= 0, s["g_top"][b, :k].double(), 0.0)
            v.scatter_add_(1, top.clamp(min=0), gt)
            g = g + gt.sum(1)
        v -= p * g[:, None]
        if s["g_entropy"] is not None:
            v -= s["g_entropy"][b, :k].double()[:, None] * torch.nan_to_num(p * (lp + H[:, None]), nan=0.0)
        grad[b, :k] = v / s["temperature"][b].double()
    return out if grad is None else grad
