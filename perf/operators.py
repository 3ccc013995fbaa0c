"""Operators around the head that can be timed and compared: 4-bit microscaled rows, the product with a 4-bit head,
log-probabilities of given tokens with their gradient, and the clipped policy loss with its gradient.

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` is one pass: in elementary
torch operations where `own` is false, through this library's entry points where it is true.  `exact` computes the same from the definitions in
float64.

A 4-bit microscaled row is cut into blocks of 32 elements.  A block has one scale 2^e, e = floor(log2 max|x|) - 2, kept as the byte
e + 127, and 32 elements x / 2^e rounded to 0, 0.5, 1, 1.5, 2, 3, 4 or 6 (ties to the even code, larger magnitudes to 6), kept as sign and
index in four bits, the even element in the low half of a byte.  Rows are padded to a multiple of 128 elements with zeros.
"""
import math

import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, op, **kw):
    c = {"op": op, **kw}
    return dict(c, name=name) if name else c


def _quantize(name, rows, d, dtype="bf16", gap=0):
    return _case(name, "quantize", rows=rows, d=d, dtype=dtype, gap=gap)


def _logits(name, V, d, B, act="bf16", out="f32", bias=True):
    return _case(name, "logits", V=V, d=d, B=B, act=act, out=out, bias=bias)


def _logprobs(name, N, V, dtype="f32", grad=False, inv_temperature=1.0, vpad=0):
    return _case(name, "logprobs", N=N, V=V, dtype=dtype, grad=grad, inv_temperature=inv_temperature, vpad=vpad)


def _policy(name, N, V, dtype="bf16", beta=0.04, clip_high=0.2, inv_temperature=1.0, skip=0.2, vpad=0):
    return _case(name, "policy", N=N, V=V, dtype=dtype, beta=beta, clip_low=0.2, clip_high=clip_high, inv_temperature=inv_temperature, skip=skip,
                 vpad=vpad)


def listed():
    return [
        # the hidden state of one decode step, rounded to four bits and back: two launches, latency only
        _quantize("quantize_b1", 1, 4096),
        # float32 rows of a wider matrix, every size odd as far as the format allows
        _quantize("quantize_ragged", 8191, 2056, dtype="f32", gap=24),
        # a whole output head
        _quantize("quantize_head", 128256, 4096),
        # one user decoding on a small head: latency
        _logits("logits_b1", 32000, 1024, 1),
        # a few users, sizes that end inside every tile, both operands in four bits
        _logits("logits_b3_ragged", 64007, 2056, 3, act="mx4", bias=False),
        # a serving batch on a large vocabulary
        _logits("logits_b32", 256000, 4608, 32),
        # scoring the tokens of finished sequences, both operands in four bits, bf16 logits for the log-probabilities
        _logits("logits_b2048", 128256, 4096, 2048, act="mx4", out="bf16"),
        # log-probability of the token one sequence has just sampled
        _logprobs("logprobs_n1", 1, 32000),
        # a scoring pass over many tokens, float32 logits, a temperature
        _logprobs("logprobs_n2048", 2048, 128256, inv_temperature=1.25),
        # a loss of the caller's own: log-probabilities and their gradient, odd sizes, the vocabulary's padding masked with -inf
        _logprobs("logprobs_grad_ragged", 509, 151669, dtype="bf16", grad=True, vpad=267),
        # a training micro-batch of a few tokens, float32 logits
        _policy("policy_n7", 7, 32003, dtype="f32", skip=0.0),
        # a training micro-batch of packed sequences, a fifth of the rows prompt or padding
        _policy("policy_n4096", 4096, 128256, clip_high=0.28),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges; sizes odd as often as not (d stays a multiple of 8)."""
    op = rng.choice(["quantize", "logits", "logprobs", "policy"])
    if op == "quantize":
        while True:
            rows, d = _log_int(rng, 1, 128256), 8 * _log_int(rng, 32, 1024)
            if rows * d <= 128256 * 4096:
                return _quantize(None, rows, d, dtype=rng.choice(["bf16", "bf16", "f32"]), gap=rng.choice([0, 0, 8, 40]))
    V = _log_int(rng, 24000, 256000)
    if op == "logits":
        while True:
            d, B = 8 * _log_int(rng, 96, 1024), _log_int(rng, 1, 2048)
            if V * d <= 256000 * 4608 and V * d * B <= 128256 * 4096 * 2048 and B * V <= 128256 * 2048:
                return _logits(None, V, d, B, act=rng.choice(["bf16", "mx4"]), out=rng.choice(["f32", "f32", "bf16"]), bias=rng.random() < 0.5)
            V = _log_int(rng, 24000, 256000)
    vpad, it, dtype = rng.choice([0, 0, 100]), rng.choice([1.0, 1.0, 1.25, 0.7]), rng.choice(["bf16", "f32"])
    most = 4096 * 128256 // (1 if dtype == "bf16" else 2)
    N = min(_log_int(rng, 1, 4096), most // V)
    if op == "logprobs":
        return _logprobs(None, N, V, dtype=dtype, grad=rng.random() < 0.5, inv_temperature=it, vpad=vpad)
    return _policy(None, N, V, dtype=dtype, beta=rng.choice([0.0, 0.04, 0.1]), clip_high=rng.choice([0.2, 0.28]), inv_temperature=it,
                   skip=rng.choice([0.0, 0.2, 0.5]), vpad=vpad)


# ------------------------------------------------------------------------------------------------ inputs
def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _head(V, d, gen):
    """Rows of a trained output matrix: normal around a few shared directions, some columns much larger than the others."""
    W = torch.randn(V, d, generator=gen, device="cuda").mul_(0.02)
    W += torch.randn(V, 1, generator=gen, device="cuda") * (0.01 * torch.randn(d, generator=gen, device="cuda"))
    W[:, torch.randperm(d, generator=gen, device="cuda")[:max(1, d // 256)]] *= 6.0
    return W


def _hidden(B, d, gen):
    """Normalised hidden states: unit variance, a few outlier channels."""
    h = torch.randn(B, d, generator=gen, device="cuda")
    h[:, torch.randperm(d, generator=gen, device="cuda")[:max(1, d // 512)]] *= 12.0
    return h.to(torch.bfloat16)


def _logit_rows(c, gen):
    """Logits [N,V] with a few likely tokens a row, the padded end of the vocabulary at minus infinity, and tokens sampled from them."""
    N, V = c["N"], c["V"]
    x = torch.randn(N, V, generator=gen, device="cuda").mul_(2.0)
    real = V - c["vpad"]
    ids = torch.randint(0, real, (N, 4), generator=gen, device="cuda")
    x.scatter_(1, ids, 9.0 + 3.0 * torch.rand(N, 4, generator=gen, device="cuda"))
    x[:, real:] = -math.inf
    pick = torch.randint(0, 4, (N, 1), generator=gen, device="cuda")
    tokens = torch.where(torch.rand(N, generator=gen, device="cuda") < 0.8, ids.gather(1, pick)[:, 0], torch.randint(0, real, (N,), generator=gen, device="cuda"))
    return x.to(_type(c["dtype"])), tokens.to(torch.int32)


def _pow2(e):
    """float64 2^e for whole numbers e (the library's pow may be off by a unit in the last place)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _pack(x):
    """Codes uint8 [R, dp/2] and scale bytes uint8 [R, dp/32] of the rows of x, dp = d rounded up to 128."""
    R, d = x.shape
    dp = -(-d // 128) * 128
    v = torch.zeros(R, dp, device=x.device)
    v[:, :d] = x
    v = v.view(R, dp // 32, 32)
    e = torch.frexp(v.abs().amax(-1)).exponent - 3
    e = torch.where(v.abs().amax(-1) == 0, torch.full_like(e, -127), e.clamp(-127, 127))
    v = v * _pow2(-e)[..., None].float()
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step).mul_(step).clamp_(max=6.0)
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, 2 + a, 4 + 0.5 * a)).to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 3)
    code = code.view(R, dp // 2, 2)
    return code[..., 0] | (code[..., 1] << 4), (e + 127).to(torch.uint8)


def prepare(case, seed):
    gen = _gen(seed)
    s = {"case": case}
    op = case["op"]
    if op == "quantize":
        x = _head(case["rows"], case["d"] + case["gap"], gen) if case["rows"] > 1 else _hidden(1, case["d"] + case["gap"], gen)
        s["x"] = x.to(_type(case["dtype"]))[:, :case["d"]]
        dp = -(-case["d"] // 128) * 128
        s["codes"] = torch.empty(case["rows"], dp // 2, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(case["rows"], dp // 32, dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty(case["rows"], case["d"], dtype=s["x"].dtype, device="cuda")
    elif op == "logits":
        V, d, B = case["V"], case["d"], case["B"]
        s["codes"], s["scales"] = _pack(_head(V, d, gen))
        s["bias"] = torch.randn(V, generator=gen, device="cuda").mul_(0.1) if case["bias"] else None
        s["h"] = _hidden(B, d, gen)
        s["out"] = torch.empty(B, V, dtype=_type(case["out"]), device="cuda")
        if own:                             # a serving program lays its head out once
            import paper_2511_21702_amd as csv
            s["head"] = csv.csv_mx4_head(s["codes"], s["scales"], s["bias"], d)
    else:
        s["logits"], s["tokens"] = _logit_rows(case, gen)
        N = case["N"]
        s["logp"] = torch.empty(N, device="cuda")
        if op == "logprobs":
            s["stats"] = torch.empty(N, 2, device="cuda")
            s["grad_logp"] = torch.randn(N, generator=gen, device="cuda") / N
        else:                               # the policy of the rollout and the reference are near the one that is trained
            logp = _plain_logp(s["logits"], s["tokens"], case["inv_temperature"])[0].float()
            s["old"] = logp + 0.15 * torch.randn(N, generator=gen, device="cuda")
            s["ref"] = logp + 0.3 * torch.randn(N, generator=gen, device="cuda") if case["beta"] > 0 else None
            s["adv"] = torch.randn(N, generator=gen, device="cuda")
            keep = torch.ones(N, device="cuda")
            keep[:int(case["skip"] * N)] = 0.0
            s["weights"] = keep / keep.sum()
            s["loss"] = torch.empty((), device="cuda")
        if op == "policy" or case["grad"]:
            s["grad"] = torch.empty_like(s["logits"])
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _values(codes, scales, d):
    """float32 values of 4-bit rows."""
    table = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    code = torch.stack((codes & 15, codes >> 4), dim=-1).view(codes.shape[0], -1).long()
    e = scales.to(torch.int32) - 127
    return (table[code].view(codes.shape[0], -1, 32) * _pow2(e)[..., None].float()).view(codes.shape[0], -1)[:, :d]


def _plain_logp(logits, tokens, c):
    """Log-probabilities (float64), exponentials and their sum (float32)."""
    x = logits.float()
    m = x.amax(1, keepdim=True)
    e = torch.exp((x - m) * c)
    total = e.sum(1, keepdim=True)
    return c * (x.gather(1, tokens.long()[:, None]).double() - m.double())[:, 0] - torch.log(total.double())[:, 0], e, total


def _plain_grad(e, total, tokens, g, c, dtype):
    """c g ([j = token] - p_j), from the exponentials and their sum."""
    g = (g * c).float()[:, None]
    out = e / total * -g
    out.scatter_add_(1, tokens.long()[:, None], g)
    return out.to(dtype)


def _policy_terms(case, logp, old, ref, adv, weights):
    """The loss and its derivative by each log-probability, all in float64."""
    old, adv, w = old.double(), adv.double(), weights.double()
    r = torch.exp(logp - old)
    lo, hi = 1.0 - case["clip_low"], 1.0 + case["clip_high"]
    term = -torch.minimum(r * adv, r.clamp(lo, hi) * adv)
    d = -adv * r * torch.where(adv >= 0, r <= hi, r >= lo)
    if ref is not None:
        k = ref.double() - logp
        term = term + case["beta"] * (torch.exp(k) - k - 1.0)
        d = d + case["beta"] * (1.0 - torch.exp(k))
    return (w * term).sum(), w * d


def run(s):
    case, op = s["case"], s["case"]["op"]
    if own:
        import paper_2511_21702_amd as csv
        if op == "quantize":
            csv.csv_mx4_quantize(s["x"], codes=s["codes"], scales=s["scales"])
            return csv.csv_mx4_dequantize(s["codes"], s["scales"], case["d"], out=s["out"])
        if op == "logits":
            return csv.csv_mx4_logits(s["head"], s["h"], out=s["out"], act=csv.ACT_MX4 if case["act"] == "mx4" else csv.ACT_BF16)
        c = case["inv_temperature"]
        if op == "logprobs":
            csv.csv_token_logprobs(s["logits"], s["tokens"], c, logp=s["logp"], stats=s["stats"])
            if not case["grad"]:
                return s["logp"]
            return [s["logp"], csv.csv_token_logprobs_backward(s["logits"], s["tokens"], s["stats"], s["grad_logp"], c, grad=s["grad"])]
        csv.csv_policy_loss(s["logits"], s["tokens"], s["old"], s["ref"], s["adv"], s["weights"], clip_low=case["clip_low"], clip_high=case["clip_high"],
                            beta=case["beta"], inv_temperature=c, loss=s["loss"], logp=s["logp"], grad=s["grad"])
        return [s["loss"], s["logp"], s["grad"]]
    if op == "quantize":
        return _values(*_pack(s["x"].float()), case["d"]).to(s["x"].dtype)
    if op == "logits":
        h = s["h"].float()
        if case["act"] == "mx4":
            h = _values(*_pack(h), case["d"])
        out = h @ _values(s["codes"], s["scales"], case["d"]).T
        return (out if s["bias"] is None else out + s["bias"]).to(_type(case["out"]))
    c = case["inv_temperature"]
    logp, e, total = _plain_logp(s["logits"], s["tokens"], c)
    if op == "logprobs":
        if not case["grad"]:
            return logp.float()
        return [logp.float(), _plain_grad(e, total, s["tokens"], s["grad_logp"], c, s["logits"].dtype)]
    loss, g = _policy_terms(case, logp, s["old"], s["ref"], s["adv"], s["weights"])
    return [loss.float(), torch.where(s["weights"] == 0, 0.0, logp).float(), _plain_grad(e, total, s["tokens"], g, c, s["logits"].dtype)]


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_rows(x):
    """The values that 4-bit microscaled rows stand for, by comparing with the powers of two and with the midpoints of the grid."""
    R, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % 32)).view(R, -1, 32)
    powers = _pow2(torch.arange(-149, 128, device=x.device))
    e = torch.searchsorted(powers, x.abs().amax(-1), right=True) - 150
    scale = _pow2((e - 2).clamp(-127, 127))[..., None]
    a = x.abs() / scale
    out = torch.zeros_like(a)
    for i in range(7):                      # at a midpoint the even one of the two codes
        mid = 0.5 * (GRID[i] + GRID[i + 1])
        out[a > mid if i % 2 == 0 else a >= mid] = GRID[i + 1]
    return (torch.copysign(out, x) * scale).view(R, -1)[:, :d]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        return _exact_rows(s["x"].double())
    if op == "logits":
        d = case["d"]
        table = torch.tensor(GRID, dtype=torch.float64, device="cuda")
        W = torch.empty(case["V"], 2 * s["codes"].shape[1], dtype=torch.float64, device="cuda")
        for half, code in enumerate((s["codes"] & 15, s["codes"] >> 4)):
            W[:, half::2] = table[(code & 7).long()] * (1.0 - 2.0 * (code >> 3).double())
        W *= _pow2(s["scales"].long() - 127).repeat_interleave(32, dim=1)
        h = s["h"].double()
        if case["act"] == "mx4":
            h = _exact_rows(h)
        out = h @ W[:, :d].T
        return out if s["bias"] is None else out + s["bias"].double()
    x, t, c = s["logits"].double() * case["inv_temperature"], s["tokens"].long()[:, None], case["inv_temperature"]
    p = torch.softmax(x, dim=1)
    logp = (x.gather(1, t) - torch.logsumexp(x, dim=1, keepdim=True))[:, 0]
    if op == "logprobs":
        if not case["grad"]:
            return logp
        loss, g = None, s["grad_logp"].double()
    else:
        # the derivative of the smaller of two products is that of the one that is smaller
        w, A, r = s["weights"].double(), s["adv"].double(), torch.exp(logp - s["old"].double())
        cut = torch.clip(r, 1.0 - case["clip_low"], 1.0 + case["clip_high"])
        loss, g = -torch.min(r * A, cut * A), torch.where(r * A <= cut * A, -r * A, 0.0)
        if s["ref"] is not None:
            k = s["ref"].double() - logp
            loss, g = loss + case["beta"] * (torch.expm1(k) - k), g - case["beta"] * torch.expm1(k)
        loss, g, logp = (loss * w).sum(), g * w, logp * (w != 0)
    p *= -c * g[:, None]
    p.scatter_add_(1, t, c * g[:, None])
    return [logp, p] if loss is None else [loss, logp, p]


# ------------------------------------------------------------------------------------------------ work
def work(case):
    """Bytes and operations of one pass that no implementation can do without."""
    op = case["op"]
    if op == "quantize":                    # rows read, codes and scales written, values written
        n, size = float(case["rows"]) * case["d"], 2.0 if case["dtype"] == "bf16" else 4.0
        return {"bytes": n * (2.0 * size + 0.5 + 1.0 / 32.0), "flops": 4.0 * n}
    if op == "logits":
        V, d, B = float(case["V"]), case["d"], case["B"]
        size = 4.0 if case["out"] == "f32" else 2.0
        return {"bytes": V * d * (0.5 + 1.0 / 32.0) + (4.0 * V if case["bias"] else 0.0) + 2.0 * B * d + size * B * V, "flops": 2.0 * V * d * B}
    n, size = float(case["N"]) * case["V"], 2.0 if case["dtype"] == "bf16" else 4.0
    if op == "logprobs":
        return {"bytes": n * size * (2.0 if case["grad"] else 1.0) + 16.0 * case["N"], "flops": n * (7.0 if case["grad"] else 4.0)}
    used = 1.0 - int(case["skip"] * case["N"]) / case["N"]
    return {"bytes": n * size * (1.0 + used) + 28.0 * case["N"], "flops": 7.0 * used * n}
