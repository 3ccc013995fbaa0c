"""What log-probabilities, policy losses and gradients are off by, on average and where the terms of a loss cancel: errors go either way, row by row.

The bounds here count a row's errors as independent of each other and of other rows' (roundings to nearest).  U = 2^-24, in units of a row's sum of
exponentials, with a the distance of a logit from the largest one in units of the exponent, p its probability:
  a term              its argument is rounded twice, 2 a U; the exponential is off by up to a unit, 2 U
  a thread's sum      up to n = V / 256 additions of U of what it holds, and 256 threads or more
  a part's sum        U where it is kept as a float32
and what all rows share, the mean error of the hardware's exponential, which is below 5e-9 over every tenth of a period (2^22 arguments in each).
A term is multiplied with two more of them on its way, where threads and parts meet.
Six standard deviations are allowed for a mean.
"""
import math

import pytest

from ._harness import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
U = 2.0 ** -24
COMMON = 5e-9


def _csv():
    import paper_2511_21702_amd as csv
    return csv


def _logits(N, V, dtype, seed):
    """Rows with a few likely tokens, and tokens that are one of those."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(N, V, generator=gen, device="cuda").mul_(2.0)
    ids = torch.randint(0, V, (N, 4), generator=gen, device="cuda")
    x.scatter_(1, ids, 11.0 + 3.0 * torch.rand(N, 4, generator=gen, device="cuda"))
    return x.to(dtype), ids[:, 0].to(torch.int32).contiguous()


def _exact(x, t, c):
    """float64: log-probabilities, log-sum-exp relative to the largest logit, and the standard deviation that a row's errors are allowed."""
    N, V = x.shape
    out = []
    for i in range(0, N, 256):
        v = x[i:i + 256].double() * c
        m = v.amax(1, keepdim=True)
        lse = torch.logsumexp(v, 1, keepdim=True)
        p, a = torch.exp(v - lse), m - v
        p2 = (p * p).sum(1)
        var = (p * p * (2 * a + 2) ** 2).sum(1) + 2 * (V / 256) * (p2 + 1 / 256) + 1
        out.append(torch.stack(((v.gather(1, t[i:i + 256].long()[:, None]) - lse)[:, 0], (lse - m)[:, 0], U * var.sqrt())))
    return torch.cat(out, 1)


def _half_step(v):
    return torch.exp2(torch.floor(torch.log2(v.abs())) - 24)


# c: as it is in float32.  Its product with log2(e) is as far from a float32 as -1.3e-8 (1.0), -5.0e-8 (0.734375) and 5.5e-8 (0.71875), relative
@pytest.mark.parametrize("c", [1.0, 0.734375, 0.71875])
@pytest.mark.parametrize("N,V,calls,dtype", [(2048, 64007, 1, F32), (2048, 64007, 1, BF16), (20, 130003, 60, F32)])
def test_errors_of_log_probabilities_go_either_way(N, V, calls, dtype, c):
    csv = _csv()
    err, serr, gerr, var, svar, gvar = [], [], [], 0.0, 0.0, 0.0
    for k in range(calls):
        if k % 20 == 0:
            log(f"log-probabilities N={N} V={V} {dtype} c={c} call {k}")
        x, t = _logits(N, V, dtype, 31 * k + 1)
        logp, stats = csv.csv_token_logprobs(x, t, c)
        want, ls, sigma = _exact(x, t, c)
        err.append(logp.double() - want)
        serr.append(torch.log(stats[:, 1].double()) - ls)
        var += (_half_step(want) ** 2 + sigma ** 2).sum().item()
        svar += (sigma ** 2).sum().item() + N * U ** 2
        if dtype == F32:            # the gradient's elements: what they are short of adding up to 0
            grad = csv.csv_token_logprobs_backward(x, t, stats, torch.ones(N, device="cuda"), c)
            gerr.append(grad.double().sum(1) / c)
            # the coefficient and its quotient by s are rounded, and every element; the token's element, near 1, too
            gvar += (2 * sigma ** 2).sum().item() + N * (3 * U) ** 2
    n = N * calls
    mean = torch.cat(err).mean().item()
    log(f"mean error of logp {mean:.2e}, of ln s {torch.cat(serr).mean().item():.2e}" + (f", of gradients {torch.cat(gerr).mean().item():.2e}" if gerr else ""))
    assert abs(mean) <= COMMON + 6 * math.sqrt(var) / n
    assert abs(torch.cat(serr).mean().item()) <= COMMON + 6 * math.sqrt(svar) / n
    if gerr:
        assert abs(torch.cat(gerr).mean().item()) <= 2 * COMMON + 6 * math.sqrt(gvar) / n


@pytest.mark.parametrize("N,V,dtype", [(2048, 64007, F32), (1500, 64007, BF16), (110, 64007, F32)])
def test_policy_loss_whose_terms_cancel(N, V, dtype):
    """Half of the rows inside the clip with advantage 1, the other half beyond it with advantage -1 and the weight that makes up for them: what is left is
    far below one term, and is still the sum's."""
    csv = _csv()
    log(f"cancelling policy loss N={N} V={V} {dtype}")
    x, t = _logits(N, V, dtype, 77)
    want, _, sigma = _exact(x, t, 1.0)
    half = N // 2
    old = want.float()
    old[half:] += 1.0                                       # a ratio of 0.37, below the clip's 0.75
    adv = torch.ones(N, device="cuda")
    adv[half:] = -1.0
    r = torch.exp(want - old.double())
    w = torch.full((N,), 1.0 / half, device="cuda")
    w[half:] = (r[:half].mean() / 0.75 / (N - half)).float()
    terms = w.double() * torch.where(adv > 0, -r, torch.full_like(r, 0.75))
    exact = terms.sum().item()
    loss = csv.csv_policy_loss(x, t, old, None, adv, w, clip_low=0.25, clip_high=0.25, want_grad=False)[0].item()
    slope = (w.double() * r)[:half]
    log(f"loss {loss:.3e} exact {exact:.3e}")
    assert abs(exact) < 1e-6
    assert abs(loss - exact) <= COMMON * slope.sum().item() + 6 * ((slope * sigma[:half]) ** 2).sum().sqrt().item() + U * abs(exact) + 1e-15


def _with_left_out(rows, values, N):
    """Vectors of N rows: the given ones first, the rest of weight 0 (the last vector)."""
    out = []
    for v, rest in values:
        t = torch.full((N,), rest, device="cuda")
        t[:rows] = torch.tensor(v, device="cuda")
        out.append(t)
    return out


@pytest.mark.parametrize("N", [2, 130])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_parameters_keep_the_digits_of_a_double(N, dtype):
    """Rows whose log-probabilities are exact, so that temperature, clip and beta are all that a loss can be off by."""
    csv = _csv()
    log(f"parameters as doubles N={N} {dtype}")
    x = torch.zeros(N, 2, dtype=dtype, device="cuda")
    x[:, 1] = -1000.0                                       # log-probability of token 1: c times that, what is added to it is below 2^-1000
    t = torch.ones(N, dtype=torch.int32, device="cuda")
    # temperature: 0.7 times 1000 is 700 to 1e-13, a ratio of 1 to as much; 0.7 as a float32 makes it 1 + 1.2e-5
    old, adv, w = _with_left_out(2, [([-700.0] * 2, 0.0), ([1.0] * 2, 0.0), ([0.5] * 2, 0.0)], N)
    loss, logp, _ = csv.csv_policy_loss(x, t, old, None, adv, w, inv_temperature=0.7)
    assert abs(loss.item() + 1.0) <= 2.0 ** -24 and logp[0].item() == -700.0
    # clip: 0.5 times 1.2 less 0.75 times 0.8, ratios far beyond either border
    old, adv, w = _with_left_out(2, [([-1002.0, -998.0], 0.0), ([1.0, -1.0], 0.0), ([0.5, 0.75], 0.0)], N)
    loss = csv.csv_policy_loss(x, t, old, None, adv, w, clip_low=0.2, clip_high=0.2)[0].item()
    assert abs(loss) <= 4 * 2.0 ** -53
    # beta: a term of 0.1 (e - 2) in both rows, and advantages that add up to them as far as two float32 can
    v = 2 * 0.1 * (math.e - 2.0)
    a0 = torch.tensor(v, dtype=F32).item()
    a1 = torch.tensor(v - a0, dtype=F32).item()
    old, ref, adv, w = _with_left_out(2, [([-1000.0] * 2, 0.0), ([-999.0] * 2, 0.0), ([a0, a1], 0.0), ([1.0] * 2, 0.0)], N)
    loss = csv.csv_policy_loss(x, t, old, ref, adv, w, beta=0.1)[0].item()
    assert abs(loss - (v - a0 - a1)) <= 16 * 2.0 ** -53


@pytest.mark.parametrize("V", [2000, 32003])
def test_a_row_that_is_cut_loses_no_digits_where_its_parts_meet(V):
    """A flat row's sum has many small errors that average out; one rounding of the whole to a float32 would be larger than all of them.  What the kernel
    holds beyond a float32 shows in a loss of two rows: the ratio of the first less a ratio of exactly 1."""
    csv = _csv()
    log(f"digits of a cut row V={V}")
    gen = torch.Generator(device="cuda").manual_seed(V)
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    w = torch.ones(2, device="cuda")
    adv = torch.tensor([1.0, -1.0], device="cuda")
    errors, var = [], 0.0
    calls = 300
    for k in range(calls):
        x = torch.randn(2, V, generator=gen, device="cuda")
        x[1] = -1000.0                                      # the second row: token 0 has a log-probability of 0
        x[1, 0] = 0.0
        want = _exact(x, t, 1.0)[0]
        old = want.float()
        loss = csv.csv_policy_loss(x, t, old, None, adv, w, want_grad=False)[0]
        errors.append(-loss.double() - torch.expm1(want[0] - old[0].double()))
        p = torch.softmax(x[0].double(), 0)
        a = x[0].double().amax() - x[0].double()
        # standard deviations: two roundings of an argument, a U / sqrt(3) each; the exponential's, 0.6 U; four of a thread's sum, 250 threads a part;
        # where threads meet in a part and parts in a row, each of them is multiplied with another exponential, and its mean error comes in again
        parts = (V - 1) // 2048 + 1
        var += ((p * p * (2 / 3 * a * a + 0.36)).sum().item() + (4 / 3 + 0.7) / (250 * parts) + (0.36 / parts if parts > 1 else 0.0)) * U ** 2
    rms = torch.stack(errors).pow(2).mean().sqrt().item()
    allowed = 1.5 * math.sqrt(var / calls) + COMMON * (3 if parts > 1 else 2)
    log(f"rms {rms:.2e}, allowed {allowed:.2e}, half a step of a float32 between 1 and 2 {U:.2e}")
    assert rms <= allowed
