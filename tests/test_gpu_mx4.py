"""4-bit microscaled rows and the product with a 4-bit head against their definitions in float64."""
import numpy as np
import pytest

from . import _operators as O
from ._harness import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F32, BF16 = torch.float32, torch.bfloat16


def _csv():
    import paper_2511_21702_amd as csv
    return csv


def _special(R, d, gen):
    """Normal rows, with blocks of zeros, subnormals, the largest values, ties of the grid, exact powers of two, and values that are not finite."""
    x = torch.randn(R, d, generator=gen) * torch.exp(3 * torch.randn(R, 1, generator=gen))
    v = x.view(-1, 8)
    n = v.shape[0]
    v[0] = 0.0
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    if n > 40:
        v[4:8] = 0.0                                    # a whole block where d is a multiple of 32
        v[9] = ties * torch.tensor([1.0, -1, 1, -1, 1, -1, 1, -1])
        v[12] = 2.0 ** torch.arange(-4, 4).float()
        v[17] = 1e-39                                   # subnormal
        v[21] = 3.38e38
        v[25, 3] = float("inf")
        v[29, 5] = float("nan")
        v[33] = -0.0
        v[37] = 2.0 ** -126
    return x


@pytest.mark.parametrize("R,d", [(1, 8), (3, 40), (17, 128), (2, 512), (5, 520), (9, 2056), (131, 136), (4099, 264), (1, 16384)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gap", [0, 24])
def test_quantize_every_code(R, d, dtype, gap):
    csv = _csv()
    log(f"quantize R={R} d={d} {dtype} gap={gap}")
    gen = torch.Generator().manual_seed(R * 7 + d)
    wide = torch.full((R, d + gap), float("nan"))       # what lies between the rows is not read
    wide[:, :d] = _special(R, d, gen)
    x = wide.to(dtype).cuda()[:, :d]
    want_c, want_s = O.mx4_quantize(O.bf16_values(x.cpu()))
    dp = O.padded(d)
    codes = torch.full((R * dp // 2 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((R * dp // 32 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    csv.csv_mx4_quantize(x, codes[:R * dp // 2].view(R, dp // 2), scales[:R * dp // 32].view(R, dp // 32))
    torch.cuda.synchronize()
    assert np.array_equal(scales.cpu().numpy()[:-64].reshape(R, -1), want_s)
    assert np.array_equal(codes.cpu().numpy()[:-64].reshape(R, -1), want_c)
    assert bool((codes[-64:] == 0xA5).all()) and bool((scales[-64:] == 0xA5).all())
    # and the values, into rows with a gap that stays as it was
    for out_type in (BF16, F32):
        out = torch.full((R, d + gap), 7.0, dtype=out_type, device="cuda")
        csv.csv_mx4_dequantize(codes[:R * dp // 2].view(R, -1), scales[:R * dp // 32].view(R, -1), d, out=out[:, :d])
        got = out.cpu().double().numpy()
        assert np.array_equal(got[:, :d], O.mx4_values(want_c, want_s, d), equal_nan=True)
        assert (got[:, d:] == 7.0).all()


@pytest.mark.parametrize("R,d", [(140003, 40), (3, 2400008)])
def test_quantize_many_rows_and_long_rows(R, d):
    """More rows than a grid has blocks for, and a row as long as a flattened matrix: pieces of 40 elements from a list, each rounded as in the list."""
    csv = _csv()
    log(f"quantize R={R} d={d}")
    gen = torch.Generator().manual_seed(R)
    base = (torch.randn(64, 40, generator=gen) * torch.exp(2 * torch.randn(64, 1, generator=gen))).to(BF16)
    if R > 1000:
        pick = torch.randint(0, 64, (R,), generator=gen)
        want_c, want_s = O.mx4_quantize(O.bf16_values(base))
        codes, scales = csv.csv_mx4_quantize(base[pick].cuda())
        assert np.array_equal(codes.cpu().numpy(), want_c[pick]) and np.array_equal(scales.cpu().numpy(), want_s[pick])
        return
    x = base.reshape(-1)[torch.arange(R * d) % 2560].reshape(R, d)
    codes, scales = csv.csv_mx4_quantize(x.cuda())
    for lo in (0, 1024, d // 128 // 2 * 128, d - d % 128):         # a stretch of 128 elements at a time
        hi = min(d, lo + 128)
        want_c, want_s = O.mx4_quantize(O.bf16_values(x[:, lo:hi]))
        assert np.array_equal(codes[:, lo // 2:lo // 2 + 64].cpu().numpy(), want_c)
        assert np.array_equal(scales[:, lo // 32:lo // 32 + 4].cpu().numpy(), want_s)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_dequantize_every_code_at_every_scale(dtype):
    csv = _csv()
    codes = torch.arange(256, dtype=torch.int64).to(torch.uint8).repeat(256, 1).cuda()          # 512 codes a row: all pairs
    scales = torch.arange(256, dtype=torch.int64).to(torch.uint8)[:, None].repeat(1, 16).cuda()
    got = csv.csv_mx4_dequantize(codes, scales, 512, dtype=dtype).cpu().double().numpy()
    want = O.mx4_values(codes.cpu().numpy(), scales.cpu().numpy(), 512)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.array_equal(np.signbit(got)[:255], np.signbit(want)[:255])


def _head(V, d, seed, bias=True):
    """A head of random codes (padding filled with rubbish), its values in float64, bias."""
    csv = _csv()
    gen = torch.Generator().manual_seed(seed)
    dp = O.padded(d)
    codes = torch.randint(0, 256, (V, dp // 2), generator=gen, dtype=torch.uint8)
    scales = torch.randint(117, 125, (V, dp // 32), generator=gen, dtype=torch.uint8)
    W = O.mx4_values(codes.numpy(), scales.numpy(), d)
    scales[:, -(-d // 32):] = 255
    b = torch.randn(V, generator=gen) if bias else None
    head = csv.csv_mx4_head(codes.cuda(), scales.cuda(), None if b is None else b.cuda(), d)
    assert (head.V, head.d) == (V, d)
    return head, W, np.zeros(V) if b is None else b.double().numpy()


def _check(head, W, b, h, act, out_type, got):
    d = W.shape[1]
    h64 = O.bf16_values(h)
    if act == 1:
        h64 = O.mx4_values(*O.mx4_quantize(h64), d)
    want = h64 @ W.T + b
    # exact products, at most dp roundings of float32 sums and the bias; then half a step of the output type
    tol = (O.padded(d) + 1) * O.U24 * (np.abs(h64) @ np.abs(W).T + np.abs(b))
    if out_type == BF16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    assert (np.abs(got.cpu().double().numpy() - want) <= tol).all()


SIZES = [(1, 8), (15, 40), (16, 128), (17, 136), (64, 520), (65, 264), (257, 2056), (1000, 1288), (4113, 96)]


@pytest.mark.parametrize("V,d", SIZES)
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("B", [1, 2, 16, 17, 33, 65, 130, 257])
def test_logits_of_a_head(V, d, act, B):
    csv = _csv()
    log(f"logits V={V} d={d} act={act} B={B}")
    head, W, b = _head(V, d, V + d, bias=B != 2)
    h = torch.randn(B, d, generator=torch.Generator().manual_seed(B)).to(BF16)
    for out_type in (F32, BF16):
        out = torch.full((B * V + 64,), 7.0, dtype=out_type, device="cuda")
        got = csv.csv_mx4_logits(head, h.cuda(), out=out[:B * V].view(B, V), act=act)
        _check(head, W, b, h, act, out_type, got)
        assert bool((out[B * V:] == 7.0).all())         # behind the last row: as it was
    head.free()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("V,d,B", [(2000, 4096, 7), (777, 8192, 40), (513, 6152, 300), (20000, 264, 64), (40007, 136, 512),
                                   (98305, 264, 9), (98307, 136, 30), (98400, 264, 61), (98320, 392, 70)])
def test_logits_of_long_rows_and_many_rows(V, d, B, act):
    csv = _csv()
    log(f"logits V={V} d={d} act={act} B={B}")
    head, W, b = _head(V, d, V + d)
    h = torch.randn(B, d, generator=torch.Generator().manual_seed(B)).to(BF16)
    _check(head, W, b, h, act, F32, csv.csv_mx4_logits(head, h.cuda(), act=act))
    _check(head, W, b, h, act, BF16, csv.csv_mx4_logits(head, h.cuda().view(torch.int16), act=act, dtype=BF16))
    head.free()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("V,d", [(3001, 1032), (50003, 520), (98400, 264)])
def test_bits_of_a_row_do_not_depend_on_the_batch(V, d, act):
    """One order of sums, whatever the tiles; scales far apart, so that sums round."""
    csv = _csv()
    gen = torch.Generator().manual_seed(d)
    dp = O.padded(d)
    codes = torch.randint(0, 256, (V, dp // 2), generator=gen, dtype=torch.uint8)
    scales = torch.randint(105, 135, (V, dp // 32), generator=gen, dtype=torch.uint8)
    head = csv.csv_mx4_head(codes.cuda(), scales.cuda(), None, d)
    h = (torch.randn(130, d, generator=gen) * torch.exp(3 * torch.randn(130, d, generator=gen))).to(BF16).cuda()
    whole = csv.csv_mx4_logits(head, h, act=act)
    for B in (1, 7, 16, 17, 32, 33, 64, 65, 100):
        log(f"V={V} d={d} B={B}")
        assert torch.equal(csv.csv_mx4_logits(head, h[:B], act=act), whole[:B])
    head.free()


@pytest.mark.parametrize("d", [64, 128, 264, 384, 512, 520, 768, 896, 1032, 1160])
@pytest.mark.parametrize("B", [66, 130])
def test_logits_of_many_hidden_states_at_every_number_of_steps(d, B):
    """Rows of one to ten steps of 128 elements, in tiles for many rows and many hidden states, one group of them and two."""
    csv = _csv()
    V = 50003
    log(f"logits V={V} d={d} B={B}")
    head, W, b = _head(V, d, d)
    h = torch.randn(B, d, generator=torch.Generator().manual_seed(B)).to(BF16)
    for out_type in (F32, BF16):
        _check(head, W, b, h, 1, out_type, csv.csv_mx4_logits(head, h.cuda(), act=1, dtype=out_type))
    head.free()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("B", [3, 80])
def test_values_that_are_not_finite_stay_in_their_row_and_column(act, B):
    csv = _csv()
    V, d = 200, 264
    gen = torch.Generator().manual_seed(4)
    dp = O.padded(d)
    codes = torch.randint(0, 256, (V, dp // 2), generator=gen, dtype=torch.uint8)
    scales = torch.randint(120, 125, (V, dp // 32), generator=gen, dtype=torch.uint8)
    scales[37, 8] = 255                                  # the last, partly filled block of a row
    scales[5] = 0                                        # a row at the smallest scale
    W = O.mx4_values(codes.numpy(), scales.numpy(), d)
    head = csv.csv_mx4_head(codes.cuda(), scales.cuda(), None, d)
    h = torch.randn(B, d, generator=gen).to(BF16)
    h[1, 7] = float("nan")
    h[2, 100] = float("inf")
    got = csv.csv_mx4_logits(head, h.cuda(), act=act).cpu().double().numpy()
    assert np.isnan(got[:, 37]).all() and np.isnan(got[1]).all()
    assert not np.isfinite(got[2, np.abs(W[:, 100]) > 0]).any()
    rows, cols = [i for i in range(B) if i not in (1, 2)], [j for j in range(V) if j != 37]
    assert np.isfinite(got[np.ix_(rows, cols)]).all()
    # logits of the row at scale 2^-127: products below float32's normal range, exact to its smallest step
    h64 = O.bf16_values(h)
    if act:
        h64 = O.mx4_values(*O.mx4_quantize(h64), d)
    want = (h64[rows] * W[5]).sum(1)
    assert np.abs(got[rows, 5] - want).max() <= dp * 2.0 ** -126
    head.free()


@pytest.mark.parametrize("V,B,act", [(16, 3, 0), (70, 20, 0), (515, 3, 1), (515, 40, 1), (515, 70, 0), (1024, 33, 0), (1999, 4100, 1), (2016, 4100, 1),
                                     (50001, 5, 0), (100015, 17, 1), (100003, 20, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_may_start_anywhere(V, B, act, dtype):
    """The place of the logits changes which stores write them, and nothing else: the same values, nothing around them touched."""
    csv = _csv()
    log(f"logits at shifts V={V} B={B} act={act} {dtype}")
    d = 40
    head, W, b = _head(V, d, V + B)
    h = torch.randn(B, d, generator=torch.Generator().manual_seed(B)).to(BF16).cuda()
    want = csv.csv_mx4_logits(head, h, act=act)
    _check(head, W, b, h.cpu(), act, F32, want)
    want = want.to(dtype)
    for shift in (0, 1, 2, 5, 8, 15, 16, 31):
        mem = torch.full((shift + B * V + 64,), 7.0, dtype=dtype, device="cuda")
        csv.csv_mx4_logits(head, h, out=mem[shift:shift + B * V].view(B, V), act=act)
        assert torch.equal(mem[shift:shift + B * V].view(B, V), want), shift
        assert bool((mem[:shift] == 7.0).all()) and bool((mem[shift + B * V:] == 7.0).all())
    head.free()


@pytest.mark.parametrize("d", [8, 40, 264, 1032])
@pytest.mark.parametrize("B", [1, 17, 33, 100])
def test_an_infinite_end_of_a_hidden_state_is_not_multiplied_with_padding(d, B):
    """An infinity in the last elements of a row meets those of W alone: the logit is that infinity with W's sign, not a NaN of 0 times it."""
    csv = _csv()
    V = 70
    gen = torch.Generator().manual_seed(d + B)
    dp = O.padded(d)
    codes = torch.randint(0, 256, (V, dp // 2), generator=gen, dtype=torch.uint8) | 0x11      # no zeros: the index of a magnitude is odd
    scales = torch.randint(117, 125, (V, dp // 32), generator=gen, dtype=torch.uint8)
    W = O.mx4_values(codes.numpy(), scales.numpy(), d)
    head = csv.csv_mx4_head(codes.cuda(), scales.cuda(), None, d)
    h = torch.randn(B, d, generator=gen).to(BF16)
    e = d - 1 - torch.arange(B) % 8
    h[torch.arange(B), e] = float("inf")
    got = csv.csv_mx4_logits(head, h.cuda()).cpu().double().numpy()
    assert (got == np.sign(W[:, e.numpy()]).T * np.inf).all()
    head.free()


def test_scales_at_both_ends_meet_in_the_product():
    csv = _csv()
    V, d, B = 64, 128, 16
    codes = torch.full((V, 64), 0x22, dtype=torch.uint8)              # all elements 1
    scales = torch.zeros((V, 4), dtype=torch.uint8)                  # 2^-127
    scales[32:] = 250                                                # 2^123
    head = csv.csv_mx4_head(codes.cuda(), scales.cuda(), None, d)
    h = torch.full((B, d), 2.0 ** 120).to(BF16)
    h[8:] = 2.0 ** -125
    for act in (0, 1):
        got = csv.csv_mx4_logits(head, h.cuda(), act=act).cpu().double().numpy()
        assert (got[:8, :32] == 2.0 ** 0).all() and (got[8:, 32:] == 2.0 ** 5).all()
        assert np.isinf(got[:8, 32:]).all()
    head.free()


def test_logits_offsets_beyond_32_bits():
    """More than 2^32 bytes of codes, and more than 2^31 logits."""
    csv = _csv()
    V, d = 1100003, 8192
    gen = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (V, d // 2), generator=gen, dtype=torch.uint8, device="cuda")
    scales = torch.full((V, d // 32), 120, dtype=torch.uint8, device="cuda")
    head = csv.csv_mx4_head(codes, scales, None, d)
    last = [0, V // 2, V - 70, V - 1]
    W = O.mx4_values(codes[last].cpu().numpy(), scales[last].cpu().numpy(), d)
    del codes, scales
    for act, B in ((0, 2), (1, 2), (0, 100), (1, 100)):
        log(f"codes beyond 32 bits, act={act} B={B}")
        h = torch.randn(B, d, generator=gen, device="cuda").to(BF16)
        got = csv.csv_mx4_logits(head, h, act=act)
        _check(head, W, np.zeros(len(last)), h.cpu(), act, F32, got[:, last])
    head.free()
    V, d, B = 140001, 8, 16385
    head, W, b = _head(V, d, 3)
    for act in (0, 1):
        log(f"logits beyond 32 bits, act={act}")
        h = torch.randn(B, d, generator=gen, device="cuda").to(BF16)
        got = csv.csv_mx4_logits(head, h, act=act, dtype=BF16)
        rows = [0, B // 2, B - 18, B - 1]
        _check(head, W, b, h[rows].cpu(), act, BF16, got[rows])
        del got
    head.free()


def test_nothing_to_do():
    csv = _csv()
    codes, scales = csv.csv_mx4_quantize(torch.empty(0, 64, device="cuda"))
    assert tuple(codes.shape) == (0, 64) and tuple(scales.shape) == (0, 4)
    assert tuple(csv.csv_mx4_dequantize(codes, scales, 64).shape) == (0, 64)
    head, _, _ = _head(17, 64, 1)
    assert tuple(csv.csv_mx4_logits(head, torch.empty(0, 64, dtype=BF16, device="cuda")).shape) == (0, 17)
    head.free()


def test_refusals_on_the_device():
    csv = _csv()
    head, _, _ = _head(40, 64, 1)
    h = torch.zeros(3, 64, dtype=BF16, device="cuda")
    with pytest.raises(ValueError):
        csv.csv_mx4_logits(head, torch.zeros(3, 72, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        csv.csv_mx4_logits(head, h.half())
    with pytest.raises(ValueError):
        csv.csv_mx4_logits(head, h, out=torch.zeros(3, 41, device="cuda"))
    with pytest.raises(ValueError):
        csv.csv_mx4_logits(head, h, out=torch.zeros(3, 40, device="cuda", dtype=torch.float16))
    with pytest.raises(csv.CsvError) as e:
        csv.csv_mx4_logits(head, h, act=2)
    assert e.value.code == -1
    with pytest.raises(csv.CsvError) as e:
        csv.csv_mx4_logits(head, torch.zeros(20, 64, dtype=BF16, device="cuda"), act=csv.ACT_MX4, scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -4 and "scratch" in str(e.value)
    with pytest.raises(csv.CsvError):
        csv.csv_mx4_logits(head, torch.zeros(csv.MX4_MAX_BATCH + 1, 64, dtype=BF16, device="cuda"), out=torch.empty(csv.MX4_MAX_BATCH + 1, 40, device="cuda"))
    head.free()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("B", [5, 200])
def test_captured_steps_and_a_stream_of_their_own(act, B):
    csv = _csv()
    V, d = 3001, 1032
    head, W, b = _head(V, d, 9)
    g0 = torch.Generator().manual_seed(2)
    hs = [torch.randn(B, d, generator=g0).to(BF16) for _ in range(3)]
    eager = [csv.csv_mx4_logits(head, h.cuda(), act=act).clone() for h in hs]
    side = torch.cuda.Stream()
    h = hs[0].cuda()
    torch.cuda.synchronize()
    got = csv.csv_mx4_logits(head, h, act=act, stream=side)
    side.synchronize()
    assert torch.equal(got, eager[0])
    # two graphs, each with scratch and output of its own, replayed in turn with eager work between
    graphs, outs, inp = [], [], []
    for _ in range(2):
        inp.append(hs[0].cuda())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(csv.csv_mx4_logits(head, inp[-1], act=act))
        graphs.append(g)
    for i in range(4):
        for k, g in enumerate(graphs):
            inp[k].copy_(hs[(i + k) % 3])
            g.replay()
        csv.csv_mx4_logits(head, hs[1].cuda(), act=act)
        torch.cuda.synchronize()
        for k in range(2):
            assert torch.equal(outs[k], eager[(i + k) % 3])
    head.free()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("B", [3, 40, 80])
@pytest.mark.parametrize("V", [200, 50003])
def test_products_below_the_normal_range_are_added_up(act, B, V):
    """Rows at the smallest scale, 2^-127: every product is subnormal or close to it, and the sums are right to float32's smallest step, 2^-149."""
    csv = _csv()
    d = 264
    log(f"subnormal products V={V} act={act} B={B}")
    gen = torch.Generator().manual_seed(V + B)
    dp = O.padded(d)
    codes = torch.randint(0, 256, (V, dp // 2), generator=gen, dtype=torch.uint8)
    scales = torch.zeros((V, dp // 32), dtype=torch.uint8)
    W = O.mx4_values(codes.numpy(), scales.numpy(), d)
    head = csv.csv_mx4_head(codes.cuda(), scales.cuda(), None, d)
    h = torch.randn(B, d, generator=gen).to(BF16)
    h[1] *= 2.0 ** -6                                    # products that are subnormal to the last one
    got = csv.csv_mx4_logits(head, h.cuda(), act=act).cpu().double().numpy()
    h64 = O.bf16_values(h)
    if act:
        h64 = O.mx4_values(*O.mx4_quantize(h64), d)
    want = h64 @ W.T
    # as everywhere, dp roundings of float32 sums; a rounding below the normal range is half a step of 2^-149
    tol = (dp + 1) * (O.U24 * (np.abs(h64) @ np.abs(W).T) + 2.0 ** -150)
    assert (np.abs(want) > 20 * tol).mean() > 0.99       # a sum that was lost would show
    assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()
    head.free()
