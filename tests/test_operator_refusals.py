"""What the operators around the head refuse, and requests for nothing: no launch, so no GPU."""
import ctypes as C
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ESHAPE = -1, -4
P = 4096                          # an address that no call may look at


@pytest.fixture(scope="module")
def csv():
    if not os.path.exists(os.path.join(ROOT, "paper_2511_21702_amd", "libcsvdecode.so")):
        import __graft_entry__
        __graft_entry__.build()
    import paper_2511_21702_amd
    return paper_2511_21702_amd


def test_rows_refused(csv):
    q, dq = csv.lib.csv_mx4_quantize, csv.lib.csv_mx4_dequantize
    for f in (lambda x, ty, ld, rows, d, c, s: q(x, ty, ld, rows, d, c, s, None), lambda x, ty, ld, rows, d, c, s: dq(c, s, rows, d, x, ty, ld, None)):
        assert f(P, csv.BF16, 64, -1, 64, P, P) == ESHAPE
        assert f(P, csv.BF16, 64, 4, 0, P, P) == ESHAPE
        assert f(P, csv.BF16, 64, 4, 60, P, P) == ESHAPE           # d is no multiple of 8
        assert f(P, csv.BF16, 64, 2 ** 30 + 1, 64, P, P) == ESHAPE
        assert f(P, csv.BF16, 2 ** 31, 4, 2 ** 30 + 8, P, P) == ESHAPE
        assert f(P, csv.BF16, 56, 4, 64, P, P) == ESHAPE           # stride below d
        assert f(P, csv.BF16, 68, 4, 64, P, P) == ESHAPE           # stride no multiple of 8
        assert f(P, 2, 64, 4, 64, P, P) == EINVAL                  # unknown type
        assert f(None, csv.BF16, 64, 4, 64, P, P) == EINVAL
        assert f(P, csv.BF16, 64, 4, 64, None, P) == EINVAL
        assert f(P, csv.BF16, 64, 4, 64, P, None) == EINVAL
        assert f(P + 8, csv.BF16, 64, 4, 64, P, P) == EINVAL       # alignment
        assert f(P, csv.BF16, 64, 4, 64, P + 4, P) == EINVAL
        assert f(P, csv.BF16, 64, 4, 64, P, P + 2) == EINVAL
        assert f(None, csv.F32, 64, 0, 64, None, None) == 0        # nothing to do


def test_head_and_logits_refused(csv):
    out = C.c_void_p(77)
    make = csv.lib.csv_mx4_head_create
    assert make(P, P, None, 16, 64, None, None) == EINVAL
    for args in ((None, P, None, 16, 64), (P, None, None, 16, 64), (P + 4, P, None, 16, 64)):
        out.value = 77
        assert make(*args, None, C.byref(out)) == EINVAL and out.value is None
    for V, d in ((0, 64), (16, 0), (16, 63), (2 ** 31 - 1, 64), (16, 2 ** 20 + 8)):
        out.value = 77
        assert make(P, P, None, V, d, None, C.byref(out)) == ESHAPE and out.value is None
    n = C.c_size_t()
    assert csv.lib.csv_mx4_logits_scratch(None, 1, 0, C.byref(n)) == EINVAL
    assert csv.lib.csv_mx4_logits(None, P, 1, 0, P, 0, None, 0, None) == EINVAL
    assert b"null head" in csv.lib.csv_last_error()
    assert csv.lib.csv_mx4_head_dims(None, None, None) == EINVAL
    csv.lib.csv_mx4_head_free(None)


def test_loss_refused(csv):
    n = C.c_size_t()
    for f in (csv.lib.csv_token_logprobs_scratch, csv.lib.csv_policy_loss_scratch):
        assert f(-1, 5, C.byref(n)) == ESHAPE
        assert f(1, 0, C.byref(n)) == ESHAPE
        assert f(1, 5, None) == EINVAL
        assert f(3, 70000, C.byref(n)) == 0 and n.value >= 24
        assert f(0, 70000, C.byref(n)) == 0 and n.value == 0
    assert csv.lib.csv_policy_loss_scratch(3, 100, C.byref(n)) == 0 and n.value >= 24
    assert csv.lib.csv_token_logprobs_scratch(3, 100, C.byref(n)) == 0 and n.value == 0
    assert csv.lib.csv_policy_loss_scratch(2 ** 31 - 1, 100, C.byref(n)) == 0 and n.value >= 8 * (2 ** 31 - 1)
    assert csv.lib.csv_token_logprobs_scratch(2 ** 31 - 1, 2 ** 31 - 1, C.byref(n)) == 0 and n.value == 0
    big = 1 << 40

    def fwd(x=P, ty=0, ld=70000, N=3, V=70000, t=P, c=1.0, logp=P, stats=P, scr=P, size=big):
        return csv.lib.csv_token_logprobs(x, ty, ld, N, V, t, c, logp, stats, scr, size, None)

    def bwd(x=P, ty=0, ld=100, N=3, V=100, t=P, stats=P, g=P, c=1.0, grad=2 * P, ldg=100):
        return csv.lib.csv_token_logprobs_backward(x, ty, ld, N, V, t, stats, g, c, grad, ldg, None)

    def pol(x=P, ty=0, ld=100, N=3, V=100, t=P, old=P, ref=P, adv=P, w=P, lo=0.2, hi=0.2, beta=0.1, c=1.0, loss=P, logp=P, grad=2 * P, ldg=100,
            scr=P, size=big, params=True):
        p = csv.PolicyParams(lo, hi, beta, c)
        return csv.lib.csv_policy_loss(x, ty, ld, N, V, t, old, ref, adv, w, C.byref(p) if params else None, loss, logp, grad, ldg, scr, size, None)

    for f in (fwd, bwd, pol):
        assert f(N=-1) == ESHAPE
        assert f(V=0) == ESHAPE
        assert f(ld=99, V=100) == ESHAPE
        assert f(ty=7) == EINVAL
        assert f(x=None) == EINVAL
        assert f(t=None) == EINVAL
        assert f(x=P + 2) == EINVAL                                # float32 at an odd half
        for c in (0.0, -1.0, float("nan"), float("inf"), 3e38):
            assert f(c=c) == EINVAL
    for f in (fwd, pol):
        assert f(scr=None) == ESHAPE
        assert f(size=8) == ESHAPE
        assert f(scr=P + 8) == EINVAL
    assert fwd(logp=None) == EINVAL and fwd(stats=None) == EINVAL
    assert fwd(x=None, t=None, N=0, logp=None, stats=None, scr=None, size=0) == 0
    for f in (bwd, pol):
        assert f(ldg=99) == ESHAPE
        assert f(grad=2 * P + 2) == EINVAL
        assert f(grad=P, ldg=104) == EINVAL                        # in place, other rows
    assert bwd(stats=None) == EINVAL and bwd(g=None) == EINVAL and bwd(grad=None) == EINVAL
    assert bwd(x=None, t=None, N=0, stats=None, g=None, grad=None) == 0
    assert pol(params=False) == EINVAL and pol(loss=None) == EINVAL
    for bad in (dict(lo=-0.1), dict(lo=1.5), dict(hi=-0.1), dict(hi=float("nan")), dict(beta=-1.0), dict(beta=float("inf")), dict(beta=float("nan")),
                dict(ref=None), dict(old=None), dict(adv=None), dict(w=None)):
        assert pol(**bad) == EINVAL, bad


def test_more_work_than_one_launch_holds_is_refused(csv):
    out, n = C.c_void_p(77), C.c_size_t()
    for V, d in ((2 ** 30, 256), (2 ** 31 - 300, 8), (131073, 2 ** 20)):
        out.value = 77
        assert csv.lib.csv_mx4_head_create(P, P, None, V, d, None, C.byref(out)) == ESHAPE and out.value is None
    N, huge = 4194304, 1 << 40
    assert csv.lib.csv_token_logprobs(P, 0, 4, N, 4, P, 1.0, P, P, P, huge, None) == ESHAPE
    assert b"4194303" in csv.lib.csv_last_error()
    assert csv.lib.csv_token_logprobs_backward(P, 0, 4, N, 4, P, P, P, 1.0, P, 4, None) == ESHAPE
    params = csv.PolicyParams(0.2, 0.2, 0.0, 1.0)
    assert csv.lib.csv_policy_loss(P, 0, 4, N, 4, P, P, None, P, P, C.byref(params), P, P, None, 0, P, huge, None) == ESHAPE
    # the longest row there is
    assert csv.lib.csv_policy_loss_scratch(1, 2 ** 31 - 1, C.byref(n)) == 0 and n.value == 8 + 8 * 64 + 8 + 8


def test_binding_refuses_host_tensors_and_wrong_types(csv):
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        csv.csv_mx4_quantize(x)
    with pytest.raises(ValueError):
        csv.csv_mx4_quantize(x.half())
    with pytest.raises(ValueError):
        csv.csv_mx4_quantize(x.t())
    with pytest.raises(ValueError):
        csv.csv_token_logprobs(x, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        csv.csv_policy_loss(x.double(), None, None, None, None, None)
    assert csv.mx4_padded(1) == 128 and csv.mx4_padded(128) == 128 and csv.mx4_padded(136) == 256


def test_policy_formula_against_differences():
    """The derivative that the kernels are held to, against central differences of the loss in float64, away from the borders of the clip."""
    from . import _operators as O
    rng = np.random.default_rng(3)
    N, V, c = 12, 23, 1.3
    x = rng.normal(size=(N, V)) * 2
    t = rng.integers(0, V, N)
    logp = O.rows_logp(x, t, c)[2]
    ratio = rng.choice([0.5, 0.7, 0.9, 1.1, 1.5], N)               # borders at 0.8 and 1.28
    old, ref = logp - np.log(ratio), logp + rng.normal(size=N) * 0.4
    adv, w = rng.normal(size=N), rng.uniform(0.1, 1, N)

    def loss(x):
        return O.policy(O.rows_logp(x, t, c)[2], old, ref, adv, w, 0.2, 0.28, 0.3)[0].sum()

    m, s, lp, p = O.rows_logp(x, t, c)
    g = O.grad_rows(p, s, t, O.policy(lp, old, ref, adv, w, 0.2, 0.28, 0.3)[1], c)
    h = 1e-5
    for i in range(N):
        for j in rng.integers(0, V, 4).tolist() + [int(t[i])]:
            xp, xm = x.copy(), x.copy()
            xp[i, j] += h
            xm[i, j] -= h
            # second differences of the loss are below 40: h^2 times that, and the cancellation of values near 1
            assert abs((loss(xp) - loss(xm)) / (2 * h) - g[i, j]) < 40 * h * h + 1e-10


def test_outputs_that_share_memory_are_refused(csv):
    """One block of a row reads what another one writes: an output may not lie in an input or in another output, by as little as a byte."""
    A = 1 << 24                                                    # addresses this far apart do not meet
    N, V = 5, 1000

    def fwd(**k):
        a = dict(x=A, t=2 * A, logp=3 * A, stats=4 * A, scr=5 * A)
        a.update(k)
        n = C.c_size_t()
        assert csv.lib.csv_token_logprobs_scratch(N, 80000, C.byref(n)) == 0 and n.value >= N * 8
        return csv.lib.csv_token_logprobs(a["x"], 0, 80000, N, 80000, a["t"], 1.0, a["logp"], a["stats"], a["scr"], 1 << 20, None)

    def bwd(ty=0, N=N, ld=V, ldg=V, **k):
        a = dict(x=A, t=2 * A, stats=3 * A, g=4 * A, grad=5 * A)
        a.update(k)
        return csv.lib.csv_token_logprobs_backward(a["x"], ty, ld, N, V, a["t"], a["stats"], a["g"], 1.0, a["grad"], ldg, None)

    def pol(ty=0, N=N, ld=V, ldg=V, beta=0.1, **k):
        a = dict(x=A, t=2 * A, old=3 * A, ref=4 * A, adv=5 * A, w=6 * A, loss=7 * A, logp=8 * A, grad=9 * A, scr=10 * A)
        a.update(k)
        p = csv.PolicyParams(0.2, 0.2, beta, 1.0)
        return csv.lib.csv_policy_loss(a["x"], ty, ld, N, V, a["t"], a["old"], a["ref"], a["adv"], a["w"], C.byref(p), a["loss"], a["logp"], a["grad"], ldg,
                                       a["scr"], 1 << 20, None)

    def refused(rc, first, second):
        assert rc == EINVAL
        assert csv.lib.csv_last_error().decode() == f"{first} overlaps {second}"

    for N_ in (5, 300):                                            # rows in parts, one block per row
        for name, at in (("d_old_logp", 3 * A), ("d_ref_logp", 4 * A), ("d_advantages", 5 * A), ("d_weights", 6 * A), ("d_tokens", 2 * A)):
            for off in (0, 4 * (N_ - 1), -4 * (N_ - 1)):
                refused(pol(N=N_, logp=at + off), "d_logp", name)
            refused(pol(N=N_, loss=at + 4), "d_loss", name)
            refused(pol(N=N_, grad=at - 4 * N_ * V + 4), "d_grad", name)
            refused(pol(N=N_, scr=at - 16), "d_scratch", name)
        refused(pol(N=N_, logp=A + 4 * V), "d_logp", "d_logits")
        refused(pol(N=N_, logp=7 * A), "d_loss", "d_logp")
        refused(pol(N=N_, logp=9 * A + 4), "d_logp", "d_grad")
        refused(pol(N=N_, loss=10 * A), "d_loss", "d_scratch")
        for f in (bwd, pol):
            for off in (4, -4, 4 * V, -4 * V, 4 * N_ * V - 4, 4 - 4 * N_ * V):
                refused(f(N=N_, grad=A + off), "d_grad", "d_logits")
            refused(f(N=N_, ty=1, grad=A + 2), "d_grad", "d_logits")
            # rows with a gap: what lies in the gap is apart, what reaches out of it is not
            for off in (4 * V - 4, 4, 4 * V + 4, 4 * (2 * V) * (N_ - 1) + 4 * V - 4, -4 * (2 * V) * (N_ - 1) + 4, -4 * (2 * V) * (N_ - 1) - 4 * V + 4):
                refused(f(N=N_, ld=2 * V, ldg=2 * V, grad=A + off), "d_grad", "d_logits")
            # other strides: some row meets one
            refused(f(N=N_, ld=2 * V, ldg=2 * V + 1, grad=A + 4 * V), "d_grad", "d_logits")
            refused(f(N=N_, ld=3 * V, ldg=V, grad=A + 4 * V), "d_grad", "d_logits")
    refused(bwd(grad=3 * A), "d_grad", "d_stats")
    refused(bwd(grad=4 * A), "d_grad", "d_grad_logp")
    refused(bwd(N=1, grad=A + 4), "d_grad", "d_logits")
    refused(fwd(logp=2 * A), "d_logp", "d_tokens")
    refused(fwd(stats=2 * A - 4), "d_stats", "d_tokens")
    refused(fwd(stats=3 * A + 16), "d_logp", "d_stats")
    refused(fwd(logp=A + 100), "d_logp", "d_logits")
    refused(fwd(scr=4 * A), "d_stats", "d_scratch")
