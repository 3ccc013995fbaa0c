"""Log-probabilities of given tokens, their gradient and the clipped policy loss against their definitions in float64."""
import numpy as np
import pytest

from . import _operators as O
from ._harness import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}             # half a step of the type, relative
TINY = {F32: 2.0 ** -126, BF16: 2.0 ** -126}           # below this a step is absolute; the exponential returns 0 there


def _csv():
    import paper_2511_21702_amd as csv
    return csv


def _rows(N, V, dtype, seed, gap=0, shift=0):
    """Logits [N, V] on the GPU as a view with `gap` elements between the rows that starts `shift` elements into its memory; tokens."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(N, V, generator=gen) * 3
    t = torch.randint(0, V, (N,), generator=gen)
    x[torch.arange(N), t] += 6 * torch.rand(N, generator=gen)
    return _place(x, dtype, gap, shift), t.to(torch.int32).cuda()


def _place(x, dtype, gap=0, shift=0, fill=float("nan")):
    N, V = x.shape
    mem = torch.full((shift + N * (V + gap) + 8,), fill, dtype=dtype, device="cuda")
    v = mem[shift:shift + N * (V + gap)].view(N, V + gap)[:, :V]
    v.copy_(x.to(dtype))
    return v


def _grad_close(got, p, s, t, g, c, rel, x, m, dtype, relg=None):
    """got against c g ([j = t] - p).  A probability carries the sum's error `rel` and, as in it, 4 U24 of its argument and one unit of the
    exponential; coefficient, quotient, product and difference are rounded to float32 (4 U24 of what they make), the result to its type.
    relg: what the coefficient itself is off by, relative."""
    want = O.grad_rows(p, s, t, g, c)
    a = np.abs(c * (np.where(np.isfinite(x), x, m[:, None]) - m[:, None]))
    cg = np.abs(c * g)[:, None]
    tol = cg * p * (rel[:, None] + (4 * a + 8) * O.U24) + (np.abs(want) + cg * (p > 0.5)) * 4 * O.U24
    tol = tol + (np.abs(want) * relg[:, None] if relg is not None else 0.0)
    tol = tol * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want) + TINY[dtype] * (1 + cg)
    with np.errstate(invalid="ignore"):
        ok = (np.abs(got - want) <= tol) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5])


SHAPES = [(1, 1), (2, 2), (3, 5), (5, 33), (4, 255), (6, 1000), (3, 4097), (300, 515), (2, 8192), (3, 32003), (2, 70001), (2, 131073), (1, 300007)]


@pytest.mark.parametrize("N,V", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gap,shift,c", [(0, 0, 1.0), (3, 1, 0.7), (8, 0, 1.25)])
def test_logprobs_and_their_gradient(N, V, dtype, gap, shift, c):
    csv = _csv()
    log(f"logprobs N={N} V={V} {dtype} gap={gap} shift={shift} c={c}")
    c = float(np.float32(c))
    x, t = _rows(N, V, dtype, N + V, gap, shift)
    logp, stats = csv.csv_token_logprobs(x, t, c)
    x64, t64 = x.cpu().double().numpy(), t.cpu().numpy()
    m, s, want, p = O.rows_logp(x64, t64, c)
    tol, rel = O.logp_tolerance(x64, m, p, c, want)
    assert (np.abs(logp.cpu().double().numpy() - want) <= tol).all()
    st = stats.cpu().double().numpy()
    assert (st[:, 0] == m).all() and (np.abs(st[:, 1] - s) <= s * (rel + O.U24)).all()
    g = torch.randn(N, generator=torch.Generator().manual_seed(N))
    g[N // 2] = 0.0 if N > 2 else g[N // 2]
    out = _place(torch.zeros(N, V), dtype, gap=5, shift=shift + (1 if gap else 0), fill=7.0)
    got = csv.csv_token_logprobs_backward(x, t, stats, g.cuda(), c, grad=out)
    _grad_close(got.cpu().double().numpy(), p, s, t64, g.double().numpy(), c, rel, x64, m, dtype)
    assert bool(out._base[-8:].eq(7.0).all())
    # into the logits' own memory, and twice: the same bits
    again, st2 = csv.csv_token_logprobs(x, t, c)
    assert torch.equal(again, logp) and torch.equal(st2, stats)
    csv.csv_token_logprobs_backward(x, t, stats, g.cuda(), c, grad=x)
    assert torch.equal(x, got)


def test_as_many_rows_as_a_call_takes():
    csv = _csv()
    N, V = csv.LOSS_MAX_ROWS, 3
    log(f"logprobs and policy loss N={N} V={V}")
    x, t = _rows(N, V, F32, 8)
    logp, stats = csv.csv_token_logprobs(x, t)
    x64, t64 = x.cpu().double().numpy(), t.cpu().numpy()
    m, s, want, p = O.rows_logp(x64, t64, 1.0)
    tol, rel = O.logp_tolerance(x64, m, p, 1.0, want)
    assert (np.abs(logp.cpu().double().numpy() - want) <= tol).all()
    g = torch.randn(N, generator=torch.Generator().manual_seed(1))
    got = csv.csv_token_logprobs_backward(x, t, stats, g.cuda())
    _grad_close(got.cpu().double().numpy(), p, s, t64, g.double().numpy(), 1.0, rel, x64, m, F32)
    # at a ratio of exactly 1 the loss is minus the sum of w A, and the gradient that of g = -w A
    w = torch.full((N,), 2.0 ** -22)
    loss, lp, grad = csv.csv_policy_loss(x, t, logp, None, g.cuda(), w.cuda())
    assert torch.equal(lp, logp)
    # the ratio is off by what rounding the old log-probability to float32 leaves
    wa = (w.double() * g.double()).numpy()
    off = np.abs(wa) * np.abs(want) * O.U24 * 1.01
    assert abs(float(loss) + wa.sum()) <= off.sum() + (abs(wa.sum()) + np.abs(wa).sum()) * O.U24
    _grad_close(grad.cpu().double().numpy(), p, s, t64, -wa, 1.0, rel, x64, m, F32, relg=np.abs(want) * O.U24 * 1.01)
    with pytest.raises(csv.CsvError):
        csv.csv_token_logprobs(torch.zeros(N + 1, 1, device="cuda"), torch.zeros(N + 1, dtype=torch.int32, device="cuda"))


def _policy_inputs(logp, N, seed, skip=True):
    rng = np.random.default_rng(seed)
    # ratios away from the clip's borders by more than what a log-probability may be off
    old = (logp - np.log(rng.choice([0.3, 0.7, 0.9, 1.0, 1.1, 1.25, 1.4, 2.0], N))).astype(np.float32)
    ref = (logp + 0.4 * rng.normal(size=N)).astype(np.float32)
    adv = rng.normal(size=N).astype(np.float32)
    w = rng.uniform(0.1, 1.0, N).astype(np.float32) / N
    if skip and N > 2:
        w[rng.random(N) < 0.3] = 0.0
        adv[0] = 0.0
    return old, ref, adv, w


def _policy_check(csv, x, t, c, lo, hi, beta, seed, dtype, in_place=False):
    N, V = x.shape
    x64, t64 = x.cpu().double().numpy(), t.cpu().numpy()
    m, s, lp, p = O.rows_logp(x64, t64, c)
    out = O.out_of_range(t64, V)
    lp = np.where(out, 0.0, lp)
    old, ref, adv, w = _policy_inputs(lp, N, seed)
    d = [torch.from_numpy(a).cuda() for a in (old, ref, adv, w)]
    before = x._base.clone().as_strided(x.shape, x.stride(), x.storage_offset())     # the same alignment: the same order of sums
    loss, logp, grad = csv.csv_policy_loss(x, t, d[0], d[1] if beta > 0 else None, d[2], d[3], lo, hi, beta, c, grad=x if in_place else None)
    terms, g = O.policy(lp, old.astype(float), ref.astype(float), adv.astype(float), w.astype(float), float(np.float32(lo)), float(np.float32(hi)), float(np.float32(beta)))
    left = out | (w == 0)
    terms, g, lp = np.where(left, 0.0, terms), np.where(left, 0.0, g), np.where(left, 0.0, lp)
    tol, rel = O.logp_tolerance(x64, m, p, c, lp)
    assert (np.abs(logp.cpu().double().numpy() - lp) <= np.where(left, 0.0, tol)).all()
    # a log-probability that is off by rel moves a term and its derivative by at most rel times |w| (|A| r + beta exp(k)) and a little
    r, k = np.exp(np.where(left, 0.0, lp - old)), np.exp(np.where(left, 0.0, ref - lp))
    slope = np.abs(w) * (np.abs(adv) * r + beta * (k + 1.0))
    assert abs(float(loss) - terms.sum()) <= (slope * rel).sum() * 1.01 + abs(terms.sum()) * O.U24 + 1e-30
    relg = np.where(g != 0, slope * rel * 1.01 / np.maximum(np.abs(g), 1e-300), 0.0)
    # the coefficient's own error moves the token's element as well
    want = O.grad_rows(p, s, t64, g, c)
    got = grad.cpu().double().numpy()
    a = np.abs(c * (np.where(np.isfinite(x64), x64, m[:, None]) - m[:, None]))
    cg = np.abs(c * g)[:, None]
    gtol = cg * p * (rel[:, None] + (4 * a + 8) * O.U24) + (np.abs(want) + cg * (p > 0.5)) * 4 * O.U24 + np.abs(want) * relg[:, None]
    gtol = gtol * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want) + TINY[dtype] * (1 + cg)
    ok = np.abs(got - want) <= gtol
    assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5])
    # the loss alone, and the same call again: the same bits
    again = csv.csv_policy_loss(before, t, d[0], d[1] if beta > 0 else None, d[2], d[3], lo, hi, beta, c)
    alone = csv.csv_policy_loss(before, t, d[0], d[1] if beta > 0 else None, d[2], d[3], lo, hi, beta, c, want_grad=False)
    assert alone[2] is None and torch.equal(again[0], loss) and torch.equal(alone[0], loss)
    assert torch.equal(again[1], logp) and torch.equal(alone[1], logp) and torch.equal(again[2], grad)


@pytest.mark.parametrize("N,V", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gap,shift,c,beta,hi,in_place", [(0, 0, 1.0, 0.0, 0.2, False), (5, 1, 0.7, 0.1, 0.28, False), (8, 0, 1.25, 0.04, float("inf"), True)])
def test_policy_loss(N, V, dtype, gap, shift, c, beta, hi, in_place):
    log(f"policy N={N} V={V} {dtype} gap={gap} shift={shift} c={c} beta={beta} hi={hi}")
    x, t = _rows(N, V, dtype, N + V, gap, shift)
    if N > 3:
        t[1], t[3] = -1, V                               # rows that are left out
    _policy_check(_csv(), x, t, float(np.float32(c)), 0.2, hi, beta, N + V, dtype, in_place)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,N", [(1000, 8), (70001, 8), (1000, 700)])
def test_masked_rows_and_values_that_are_not_finite(dtype, V, N):
    csv = _csv()
    x, t = _rows(N, V, dtype, 5)
    inf, low = float("inf"), torch.finfo(dtype).min
    x[0, V // 2:] = -inf
    t[0] = 3
    x[1] = -inf                                          # nothing is left
    x[2, :] = low                                        # the lowest value everywhere: uniform
    x[3, ::2] = low
    t[3] = 1
    x[4, 9] = inf
    x[5, V - 1] = float("nan")
    x[6, 11] = -inf
    t[6] = 11                                            # the token itself is masked
    t[7] = -1
    logp, stats = csv.csv_token_logprobs(x, t)
    x64, t64 = x.cpu().double().numpy(), t.cpu().numpy()
    m, s, want, p = O.rows_logp(x64, t64, 1.0)
    got = logp.cpu().double().numpy()
    assert np.isneginf(got[1]) and np.isneginf(got[6]) and np.isnan(got[[4, 5]]).all() and got[7] == 0.0
    fine = [i for i in range(N) if i not in (1, 4, 5, 6, 7)]
    tol, rel = O.logp_tolerance(x64[fine], m[fine], p[fine], 1.0, want[fine])
    assert (np.abs(got[fine] - want[fine]) <= tol).all()
    g = torch.linspace(0.5, 1.5, N, device="cuda")
    grad = csv.csv_token_logprobs_backward(x, t, stats, g).cpu().double().numpy()
    assert (grad[[1, 7]] == 0).all() and np.isnan(grad[[4, 5]]).all()
    assert (grad[0, V // 2:] == 0).all()
    keep = fine + [6]
    _grad_close(grad[keep], p[keep], s[keep], t64[keep], g.cpu().double().numpy()[keep], 1.0, np.append(rel, 600 * O.U24), x64[keep], m[keep], dtype)
    # the policy loss: rows 4 and 5 by weight, 7 by token left out; row 1 has no gradient
    w = torch.full((N,), 1.0 / N, device="cuda")
    w[[4, 5]] = 0.0
    adv = torch.ones(N, device="cuda")
    old = torch.where(torch.isfinite(logp), logp, torch.zeros_like(logp))
    loss, lp, grad = csv.csv_policy_loss(x, t, old, None, adv, w)
    assert bool(torch.isfinite(loss)) and bool((grad[[1, 4, 5, 7]] == 0).all()) and bool(torch.isfinite(grad.float()).all())
    assert np.isneginf(float(lp[1])) and bool((lp[[4, 5, 7]] == 0).all())
    assert bool((grad[6] == 0).all())                    # ratio 0: no push either way
    w[4] = 1.0 / N
    loss, lp, grad = csv.csv_policy_loss(x, t, old, None, adv, w)
    assert bool(torch.isnan(loss)) and bool(torch.isnan(grad[4].float()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,V", [(6, 5003), (6, 90001), (300, 5003)])
@pytest.mark.parametrize("offset,mask,c", [(0.0, -1e4, 1.0), (0.0, -1e9, 1.3), (3e5, -1e30, 1.0), (-3e5, -1e9, 0.7), (1e6, -1e6, 1.0), (-2e8, -1e30, 1.0), (1e30, 0.0, 1e-29)])
def test_logits_far_from_zero_and_masks_by_addition(dtype, N, V, offset, mask, c):
    """Most of every row far below, by a number that is added, and rows whose largest logit is far from zero on either side."""
    csv = _csv()
    log(f"far rows N={N} V={V} {dtype} offset={offset} mask={mask}")
    c = float(np.float32(c))
    gen = torch.Generator().manual_seed(7)
    x = torch.randn(N, V, generator=gen) * (2 if abs(offset) < 1e29 else 1e29) + offset
    x[:, V // 3:] += mask
    t = torch.randint(0, V // 3, (N,), generator=gen)
    x = _place(x, dtype, gap=3, shift=1)
    t = t.to(torch.int32).cuda()
    logp, stats = csv.csv_token_logprobs(x, t, c)
    x64, t64 = x.cpu().double().numpy(), t.cpu().numpy()
    m, s, want, p = O.rows_logp(x64, t64, c)
    tol, rel = O.logp_tolerance(x64, m, p, c, want)
    assert (np.abs(logp.cpu().double().numpy() - want) <= tol).all()
    st = stats.cpu().double().numpy()
    assert (st[:, 0] == m).all() and (np.abs(st[:, 1] - s) <= s * (rel + O.U24)).all()
    g = torch.linspace(-1, 1, N)
    grad = csv.csv_token_logprobs_backward(x, t, stats, g.cuda(), c).cpu().double().numpy()
    _grad_close(grad, p, s, t64, g.double().numpy(), c, rel, x64, m, dtype)
    _policy_check(csv, x, t, c, 0.2, 0.28, 0.05, N + V, dtype)


def test_no_rows():
    csv = _csv()
    e = torch.empty(0, device="cuda")
    loss, logp, grad = csv.csv_policy_loss(torch.empty(0, 50, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), e, None, e, e,
                                           loss=torch.full((), 9.0, device="cuda"))
    assert float(loss) == 0.0 and logp.numel() == 0 and tuple(grad.shape) == (0, 50)
    logp, stats = csv.csv_token_logprobs(torch.empty(0, 50, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
    assert logp.numel() == 0
    csv.csv_token_logprobs_backward(torch.empty(0, 50, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), stats, e)


@pytest.mark.parametrize("N", [5, 200])
def test_inputs_of_a_row_that_are_not_numbers_show_in_its_gradient_alone(N):
    csv = _csv()
    V = 3001
    x, t = _rows(N, V, F32, 4)
    base, _ = csv.csv_token_logprobs(x, t)
    nan = float("nan")
    for k in range(4):                                   # old_logp, ref_logp, advantages, weights
        v = [base.clone(), base.clone(), torch.ones(N, device="cuda"), torch.full((N,), 1.0 / N, device="cuda")]
        v[k][2] = nan
        for ratio in (0.0, 1.0, -1.0):                   # on both sides of the clip
            old = v[0] - ratio
            loss, logp, grad = csv.csv_policy_loss(x, t, old, v[1], v[2], v[3], beta=0.1)
            assert bool(torch.isnan(loss)) and bool(torch.isnan(grad[2]).all()) and bool(torch.isfinite(logp).all())
            assert bool(torch.isfinite(grad[[i for i in range(N) if i != 2]]).all())


def test_all_rows_left_out():
    csv = _csv()
    x = torch.full((5, 4099), float("nan"), device="cuda")
    z = torch.zeros(5, device="cuda")
    loss, logp, grad = csv.csv_policy_loss(x, torch.zeros(5, dtype=torch.int32, device="cuda"), z, z, z, z, beta=0.1)
    assert float(loss) == 0.0 and bool((logp == 0).all()) and bool((grad == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_beyond_32_bits(dtype):
    """More than 2^31 elements (and 2^32 bytes) of logits: the last rows are right, and the first."""
    csv = _csv()
    N, V = 17000, 130003
    log(f"policy beyond 32 bits {dtype}")
    x = torch.zeros(N, V, dtype=dtype, device="cuda")
    t = torch.full((N,), 7, dtype=torch.int32, device="cuda")
    rows = [0, N - 2, N - 1]
    small, ts = _rows(3, V, dtype, 8)
    x[rows], t[rows] = small, ts
    w = torch.zeros(N, device="cuda")
    w[rows] = torch.tensor([0.5, -0.25, 1.0], device="cuda")
    one = torch.ones(N, device="cuda")
    x64, t64, w64 = small.cpu().double().numpy(), ts.cpu().numpy(), w[rows].cpu().double().numpy()
    m, s, lp, p = O.rows_logp(x64, t64, 1.0)
    tol, rel = O.logp_tolerance(x64, m, p, 1.0, lp)
    # a clip of 1 and plus infinity: the loss is -w r A, its derivative -w A r, and both carry rel of the log-probability
    loss, logp, grad = csv.csv_policy_loss(x, t, -one, None, one, w, clip_low=1.0, clip_high=float("inf"), grad=x)
    assert (np.abs(logp[rows].cpu().double().numpy() - lp) <= tol).all()
    term, g = O.policy(lp, -np.ones(3), None, np.ones(3), w64, 1.0, np.inf, 0.0)
    assert abs(float(loss) - term.sum()) <= (np.abs(term) * rel).sum() * 1.01 + abs(term.sum()) * O.U24
    _grad_close(grad[rows].cpu().double().numpy(), p, s, t64, g, 1.0, 2.01 * rel, x64, m, dtype, relg=1.01 * rel)
    assert not bool(grad[1:N - 2].any())


@pytest.mark.parametrize("N,V,dtype", [(3, 50021, F32), (700, 5003, BF16)])
def test_captured_calls_and_a_stream_of_their_own(N, V, dtype):
    csv = _csv()
    c = 1.0
    xs = [_rows(N, V, dtype, k)[0].contiguous() for k in range(3)]
    t = _rows(N, V, dtype, 0)[1]
    old = torch.full((N,), -5.0, device="cuda")
    adv = torch.linspace(-1, 1, N, device="cuda")
    w = torch.full((N,), 1.0 / N, device="cuda")

    def both(x, stream=None):
        loss, logp, grad = csv.csv_policy_loss(x, t, old, old, adv, w, beta=0.1, inv_temperature=c, stream=stream)
        lp, stats = csv.csv_token_logprobs(x, t, c, stream=stream)
        return [loss, logp, grad, lp, csv.csv_token_logprobs_backward(x, t, stats, adv, c, stream=stream)]

    eager = [[v.clone() for v in both(x)] for x in xs]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = both(xs[1], stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, eager[1]))
    inp = [xs[0].clone() for _ in range(2)]
    graphs, outs = [], []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(both(inp[k]))
        graphs.append(g)
    for i in range(4):
        for k in range(2):
            inp[k].copy_(xs[(i + k) % 3])
            graphs[k].replay()
        both(xs[2])
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[k], eager[(i + k) % 3]))


def test_rollout_head_in_four_bits_then_policy_loss_on_the_exact_head():
    """The operators in the order of a training step: the head in four bits samples and scores, the exact head's logits are trained against it."""
    csv = _csv()
    V, d, N = 2003, 264, 24
    gen = torch.Generator(device="cuda").manual_seed(6)
    W = (torch.randn(V, d, generator=gen, device="cuda") * 0.15).to(BF16)
    b = torch.randn(V, generator=gen, device="cuda") * 0.1
    h = torch.randn(N, d, generator=gen, device="cuda").to(BF16)
    idx = csv.csv_build_index(W, b, 8)
    ws = csv.CsvWorkspace(idx, N, V)
    full = csv.csv_full_logits(ws, idx, h)
    codes, scales = csv.csv_mx4_quantize(W)
    head = csv.csv_mx4_head(codes, scales, b, d)
    roll = csv.csv_mx4_logits(head, h)
    tokens = roll.argmax(1).to(torch.int32)
    old, _ = csv.csv_token_logprobs(roll, tokens)
    ref, _ = csv.csv_token_logprobs(csv.csv_mx4_logits(head, h, act=csv.ACT_MX4), tokens)
    adv = torch.randn(N, generator=gen, device="cuda")
    w = torch.full((N,), 1.0 / N, device="cuda")
    loss, logp, grad = csv.csv_policy_loss(full, tokens, old, ref, adv, w, beta=0.05)
    # the same from the operators' definitions, step by step from what the previous step gave
    c64, s64 = O.mx4_quantize(O.bf16_values(W.cpu()))
    assert np.array_equal(codes.cpu().numpy(), c64) and np.array_equal(scales.cpu().numpy(), s64)
    W4 = O.mx4_values(c64, s64, d)
    h64 = O.bf16_values(h.cpu())
    want = h64 @ W4.T + b.cpu().double().numpy()
    assert np.abs(roll.cpu().double().numpy() - want).max() <= 400 * O.U24 * (np.abs(h64) @ np.abs(W4).T).max()
    x64, t64 = full.cpu().double().numpy(), tokens.cpu().numpy()
    m, s, lp, p = O.rows_logp(x64, t64, 1.0)
    terms, g = O.policy(lp, *[v.cpu().double().numpy() for v in (old, ref, adv, w)], float(np.float32(0.2)), float(np.float32(0.2)), float(np.float32(0.05)))
    assert np.abs(logp.cpu().double().numpy() - lp).max() < 1e-5
    assert abs(float(loss) - terms.sum()) < 1e-4
    wantg = O.grad_rows(p, s, t64, g, 1.0)
    r = np.exp(lp - old.cpu().double().numpy())
    clear = (np.abs(r - 0.8) > 1e-3) & (np.abs(r - 1.2) > 1e-3)
    assert clear.sum() > N // 2 and np.abs(grad.cpu().double().numpy() - wantg)[clear].max() < 1e-5
    ws.free()
    idx.free()
    head.free()


@pytest.mark.parametrize("N,V", [(3, 80003), (130, 5000), (1, 4097)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_outputs_may_lie_between_the_rows_of_the_logits(N, V, dtype):
    """One buffer of rows: logits, their gradient beside them, and the log-probabilities behind both in the first row's gap."""
    csv = _csv()
    log(f"side by side N={N} V={V} {dtype}")
    x, t = _rows(N, V, dtype, 3)
    old, adv, w = torch.full((N,), -4.0, device="cuda"), torch.linspace(-1, 1, N, device="cuda"), torch.full((N,), 1.0 / N, device="cuda")
    gap = 2 * N + 8                                      # bfloat16 elements or more for N float32, wherever they start
    wide = torch.full((N, 2 * V + gap), 7.0, dtype=dtype, device="cuda")
    wide[:, :V] = x
    at = wide[0, 2 * V:]
    at = at[(-(at.data_ptr() // at.element_size())) % (4 // at.element_size()):]
    logp = at[:4 * N // at.element_size()].view(F32)
    assert logp.numel() == N
    loss, _, grad = csv.csv_policy_loss(wide[:, :V], t, old, None, adv, w, logp=logp, grad=wide[:, V:2 * V])
    # the same alignment of the rows: the same order of sums
    same = wide.clone()
    want = csv.csv_policy_loss(same[:, :V], t, old, None, adv, w, grad=same.new_empty(N, 2 * V + gap)[:, V:2 * V])
    assert torch.equal(loss, want[0]) and torch.equal(logp, want[1]) and torch.equal(grad, want[2])
    assert torch.equal(wide[:, :V], x)
    lp, stats = csv.csv_token_logprobs(wide[:, :V], t)
    wide[:, V:2 * V] = 7.0
    got = csv.csv_token_logprobs_backward(wide[:, :V], t, stats, adv, grad=wide[:, V:2 * V])
    assert torch.equal(got, csv.csv_token_logprobs_backward(same[:, :V], t, stats, adv, grad=same.new_empty(N, 2 * V + gap)[:, V:2 * V]))
    assert torch.equal(wide[:, :V], x)
    with pytest.raises(csv.CsvError, match="d_logp overlaps d_old_logp"):
        csv.csv_policy_loss(x, t, old, None, adv, w, logp=old)
    with pytest.raises(csv.CsvError, match="d_grad overlaps d_logits"):
        csv.csv_policy_loss(wide[:, :V], t, old, None, adv, w, grad=wide[:, V - 1:2 * V - 1])


@pytest.mark.parametrize("N,V", [(12, 1003), (12, 80003), (200, 1003)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("beta", [0.0, 0.1])
def test_policy_loss_of_masked_rows_and_masked_tokens(N, V, dtype, beta):
    """Rows that a mask leaves nothing of, tokens that are masked themselves, and what they were scored with: minus infinity too."""
    csv = _csv()
    log(f"masked rows and tokens N={N} V={V} {dtype} beta={beta}")
    x, t = _rows(N, V, dtype, 9)
    t[:] = torch.where(t < V // 2, t, t - V // 2)
    x[:, V // 2 + 1:] = -float("inf")                    # masked in every row
    x[1] = -float("inf")                                 # nothing left
    x[2] = -float("inf")
    t[3:6] = V - 1                                       # the token is masked
    old, _ = csv.csv_token_logprobs(x, t)
    assert bool(torch.isneginf(old[1:6]).all()) and bool(torch.isfinite(old[6:]).all())
    ref = old + 0.25
    old[2], old[4], ref[2] = -3.0, -3.0, -3.0            # scored as if they were not
    adv = torch.linspace(-1.0, 1.5, N, device="cuda")
    adv[3], adv[4], adv[5], adv[6], adv[7] = 0.5, -2.0, -1.0, 0.0, 1.0
    old[6] = -900.0                                      # a ratio beyond the largest double, advantage 0
    old[7] = -float("inf")                               # and plus infinity, clipped
    w = torch.full((N,), 1.0 / N, device="cuda")
    loss, logp, grad = csv.csv_policy_loss(x, t, old, ref, adv, w, clip_low=0.25, clip_high=0.5, beta=beta)
    assert bool(torch.isneginf(logp[1:6]).all())
    assert bool((grad[1:6] == 0).all()) and bool(torch.isfinite(grad.float()).all()) and bool((grad[:, V // 2 + 1:] == 0).all())
    # the same from the definition: rows 1 and 2 add nothing, 3 to 5 a ratio of 0 (advantage below 0: the clip's border), row 6 its KL term alone
    x64, t64, A = x.cpu().double().numpy(), t.cpu().numpy(), adv.cpu().double().numpy()
    m, s, lp, p = O.rows_logp(x64, t64, 1.0)
    rest = [0] + list(range(8, N))
    o64, r64 = old.cpu().double().numpy(), ref.cpu().double().numpy()
    terms = np.zeros(N)
    terms[rest] = O.policy(lp[rest], o64[rest], r64[rest], A[rest], 1.0, 0.25, 0.5, beta)[0]
    terms[4], terms[5], terms[7] = 0.75 * 2.0, 0.75 * 1.0, -1.5
    for i in (6, 7):
        k = r64[i] - lp[i]
        terms[i] += beta * (np.exp(k) - k - 1)
    slope = np.abs(A) * 1.01 + beta * 0.3                # ratios are 1, k is 0.25
    rel = np.zeros(N)
    rel[rest + [6, 7]] = O.logp_tolerance(x64[rest + [6, 7]], m[rest + [6, 7]], p[rest + [6, 7]], 1.0, lp[rest + [6, 7]])[1]
    w1 = float(w[0])
    # old and ref are rounded to float32 and known; w is what the kernel reads
    assert abs(float(loss) - w1 * terms.sum()) <= w1 * (slope * rel).sum() * 1.01 + abs(w1 * terms.sum()) * O.U24 + 1e-12
    assert bool((grad[6] == 0).all()) if beta == 0 else bool(grad[6].any())
    alone = csv.csv_policy_loss(x, t, old, ref, adv, w, clip_low=0.25, clip_high=0.5, beta=beta, want_grad=False)[0]
    assert torch.equal(alone, loss)
    if beta > 0:                                         # the reference knows a token that the policy has masked
        ref[3] = -3.0
        loss, logp, grad = csv.csv_policy_loss(x, t, old, ref, adv, w, clip_low=0.25, clip_high=0.5, beta=beta)
        assert float(loss) == float("inf") and bool((grad[3] == 0).all()) and bool(torch.isfinite(grad.float()).all())
    # a token that was masked when it was scored, is not now, and is not wanted
    adv[7] = -1.0
    loss, logp, grad = csv.csv_policy_loss(x, t, old, old if beta == 0 else ref, adv, w, clip_low=0.25, clip_high=0.5, beta=beta)
    assert float(loss) == float("inf") and bool(torch.isfinite(grad[8:].float()).all()) and not bool(torch.isfinite(grad[7].float()).all())


@pytest.mark.parametrize("N,V", [(17000, 130003), (100, 22000003)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_zeros_of_left_out_rows_beyond_32_bits(N, V, dtype):
    """More than 2^31 logits, all of them NaN in rows that are left out: each of their gradient's elements is written."""
    csv = _csv()
    log(f"zeros beyond 32 bits N={N} V={V} {dtype}")
    x = torch.full((N, V), float("nan"), dtype=dtype, device="cuda")
    t = torch.full((N,), 7, dtype=torch.int32, device="cuda")
    w, z = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")
    x[N // 2] = 0.0                                      # one row counts: its gradient is that of a uniform distribution
    w[N // 2] = 1.0
    loss, logp, grad = csv.csv_policy_loss(x, t, z - float(np.log(V)), None, z + 1.0, w, grad=x)
    assert abs(float(loss) + 1.0) < 1e-4
    rows = [i for i in range(0, N, 1000 if N > 1000 else 1)]
    assert all(not bool(grad[i:min(i + 1000, N // 2)].any()) for i in rows if i < N // 2)
    assert all(not bool(grad[max(i, N // 2 + 1):i + 1000].any()) for i in rows)
    assert bool((grad[N // 2] != 0).all())
    # the gradient of log-probabilities alone: rows with a gradient of 0 are zeros
    x.fill_(float("nan"))
    stats = torch.ones(N, 2, device="cuda")
    stats[:, 0] = 0.0
    stats[:, 1] = float(V)
    x[N - 1] = 0.0
    g = z.clone()
    g[N - 1] = 1.0
    grad = csv.csv_token_logprobs_backward(x, t, stats, g, grad=x)
    assert all(not bool(grad[i:min(i + 1000, N - 1)].any()) for i in rows)
    assert bool((grad[N - 1] != 0).all())
    del x, grad
    torch.cuda.empty_cache()


@pytest.mark.parametrize("N", [111, 112, 143, 144])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [4099, 40009])
def test_policy_loss_on_both_sides_of_the_rows_that_are_cut(N, V, dtype):
    log(f"policy N={N} V={V} {dtype}")
    x, t = _rows(N, V, dtype, N, gap=3, shift=1)
    t[N - 1] = -1
    _policy_check(_csv(), x, t, 1.0, 0.2, 0.28, 0.05, N + V, dtype)


@pytest.mark.parametrize("N,V", [(64, 125000), (64, 126000), (111, 171000), (1, 65000), (1, 67000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_log_probabilities_on_both_sides_of_the_rows_that_are_cut(N, V, dtype):
    csv = _csv()
    log(f"logprobs N={N} V={V} {dtype}")
    x, t = _rows(N, V, dtype, N, gap=1, shift=1)
    logp, stats = csv.csv_token_logprobs(x, t)
    x64, t64 = x.cpu().double().numpy(), t.cpu().numpy()
    m, s, want, p = O.rows_logp(x64, t64, 1.0)
    tol, rel = O.logp_tolerance(x64, m, p, 1.0, want)
    assert (np.abs(logp.cpu().double().numpy() - want) <= tol).all()
    st = stats.cpu().double().numpy()
    assert (st[:, 0] == m).all() and (np.abs(st[:, 1] - s) <= s * (rel + O.U24)).all()
