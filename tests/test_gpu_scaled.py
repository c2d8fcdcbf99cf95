"""The operators on 8-bit rows (include/spark.h, spark_scaled_*) against the same in 64 bits.

Rows and norm are worked out so that every code is the formula's: they are compared bit by bit.

Products with an output in fp32 are sums in fp32: each block of 128 is taken to be off by at most 2^-22 (four
fp32 half steps) of the magnitudes it adds, and so is each joining of up to 16 parts: an output of `blocks`
is off by at most (blocks + 17) 2^-22 of the sum of magnitudes, and by half a step of its type, 2^-24.

With an output in bf16 the instruction cuts each product 13 bits below the largest of its eight, seven
of them at most: 2^-10 of the eights' magnitudes, and the sums of its sixteen eights are added with 2^-24 each:
(2^-10 + 2^-20 blocks) of the magnitudes, and half a step of the type, 2^-8.

For outputs in fp32 and for pairs the weights are fp16 numbers times their row's largest power P: what lies below
2^-14 P there is held to half a step of 2^-24 P, which is only of account in rows of very different blocks.

Gated: the two sums as in fp32, silu's slope is at most 1.1, and the fp32 exponential, division and
products add at most 16 half steps; the code lies between the codes of both ends of that interval.  The sums
are some 1e-7 off and neighbouring codes 2^-3 or less apart, so that few codes lie so near to a middle that they may
differ from those of the 64-bit result: of many no more than 0.1 %."""
import pytest
import torch

import scaled_ref as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2603_09215_amd import scaled
    return scaled


def activations(m, k, seed, dtype=F32, spread=30.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, k, generator=g) * torch.exp(torch.randn(m, 1, generator=g))
    x[:, torch.rand(k, generator=g) < 0.01] *= spread
    return x.to(dtype)


def weights(n, k, seed, dtype=BF16):
    return (torch.randn(n, k, generator=torch.Generator().manual_seed(seed)) * 0.02).to(dtype)


def bits(t):
    return t.contiguous().view(torch.uint8).cpu()


def same_rows(rows, codes, powers, what=""):
    got, want = bits(rows.codes), codes
    nan = ((got & 127) == 127) & ((want & 127) == 127)   # (a NaN's sign is no part of the format)
    assert torch.equal(torch.where(nan, 0, got), torch.where(nan, 0, want)), what
    assert torch.equal(bits(rows.scales), powers), what


# ---------------------------------------------------------------------------------- rows

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k", [(1, 1), (1, 7), (3, 127), (2, 128), (5, 129), (1, 3584), (17, 1000), (33, 4100), (300, 515), (4, 18944)])
def test_rows_are_the_formulas(ops, m, k, dtype):
    x = activations(m, k, 7 * m + k, dtype)
    same_rows(ops.scaled_rows(x.cuda()), *ref.quantise(x.double()))


def test_rows_of_special_values(ops):
    x = torch.zeros(12, 256)
    x[1] = 448.0                                        # exactly at the end of the range
    x[2] = torch.nextafter(torch.tensor(448.0), torch.tensor(1e9))
    x[3] = torch.linspace(-1, 1, 256) * 3.0e38          # near fp32's end
    x[4] = torch.linspace(-1, 1, 256) * 1e-38           # near its other end
    x[5] = torch.linspace(0, 1, 256) * 1e-44            # denormal
    x[6] = torch.tensor([float("nan"), 1.0, -2.0, float("inf"), -float("inf"), 3.3, 0.0, -0.0] * 32)
    x[7] = float("nan")
    x[8] = float("inf")
    x[9, 5] = 1.0                                       # one value alone, zeros beside it
    x[10] = torch.arange(256) * 0.0625 + 0.03125        # middles between codes
    x[11] = -torch.arange(256) * 2.0 ** -10             # middles below the smallest normal code
    x[11, 0] = 448.0
    for dtype in (F32, BF16):
        t = x.to(dtype)
        same_rows(ops.scaled_rows(t.cuda()), *ref.quantise(t.double()), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_code_and_every_middle(ops, dtype):
    """all 126 steps: the codes themselves, the middles, and the neighbours of the middles (fp32)"""
    mid = (ref.TABLE[1:] + ref.TABLE[:-1]) / 2
    one = torch.cat([ref.TABLE, mid]).float()
    x = torch.cat([one, torch.nextafter(one, torch.tensor(1e9)), torch.nextafter(one, torch.tensor(-1e9))]).clamp(0, 448)
    x = torch.nn.functional.pad(x, (0, -len(x) % 127)).view(-1, 127)
    x = torch.cat([torch.full((x.shape[0], 1), 448.0), x], 1).to(dtype)   # the first holds the power at 1
    x = torch.cat([x, -x])
    same_rows(ops.scaled_rows(x.cuda()), *ref.quantise(x.double()))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(0, 8), (1, 3), (8, 24)])
def test_rows_of_a_strided_view(ops, dtype, offset, extra):
    big = activations(9, 640 + extra + offset, 3, dtype).cuda()
    x = big[:, offset:offset + 640]
    same_rows(ops.scaled_rows(x), *ref.quantise(x.cpu().double()))


def test_rows_of_many_rows(ops):
    x = activations(70000, 128, 11, BF16)
    same_rows(ops.scaled_rows(x.cuda()), *ref.quantise(x.double()))


# ---------------------------------------------------------------------------------- norm

def norm_case(ops, h, y, gain, eps, h_out=None):
    want_h, v = ref.norm(h, y, gain, eps)
    dev = h.cuda()
    rows = ops.scaled_norm(dev, gain.cuda(), eps, y=None if y is None else y.cuda(), h_out=h_out)
    got_h = (dev if h_out is None else h_out).cpu()
    assert torch.equal(got_h.double(), want_h) or torch.equal(torch.isnan(got_h.double()), torch.isnan(want_h))
    same_rows(rows, *ref.quantise(v))


@pytest.mark.parametrize("m,k", [(1, 1), (1, 64), (3, 130), (2, 2048), (5, 2500), (1, 3584), (9, 4096), (4, 4104), (2, 9000), (3, 18944), (2, 40000), (600, 256)])
@pytest.mark.parametrize("dtype,ytype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32), (F32, None), (BF16, None)])
def test_norm_is_the_formula(ops, m, k, dtype, ytype):
    h = activations(m, k, m + k, dtype)
    y = None if ytype is None else activations(m, k, m + k + 1, ytype, 1.0)
    gain = 1 + 0.1 * torch.randn(k, generator=torch.Generator().manual_seed(k))
    norm_case(ops, h, y, gain, 1e-6)


def test_norm_keeps_the_input_where_an_output_is_given(ops):
    h, y = activations(7, 1000, 1).cuda(), activations(7, 1000, 2).cuda()
    before, out = h.clone(), torch.empty_like(h)
    ops.scaled_norm(h, torch.ones(1000, device="cuda"), 1e-6, y=y, h_out=out)
    assert torch.equal(h, before) and torch.equal(out, before + y)


@pytest.mark.parametrize("ytype", [F32, BF16])
def test_bf16_sums_beside_the_middles(ops, ytype):
    """h + y at the middle between two bf16 numbers and a little beside it, further down than an fp32 sum can hold"""
    h = torch.tensor([256.0, 258.0, 1.0, -3.0, 2.0 ** -126, 1e30]).repeat_interleave(64)
    unit = 2.0 ** (torch.frexp(h.abs())[1].float() - 9)                     # half a step of bf16 at h
    off = torch.cat([torch.tensor([0.0, 1.0, -1.0]), 2.0 ** -torch.arange(7.0, 35.0), -2.0 ** -torch.arange(7.0, 35.0), torch.zeros(5)]).repeat(6)
    rows = torch.stack([h, h, h, h, h])
    y = torch.stack([unit * (1 + off), -unit * (1 + off), unit * 0.5 * (1 + off), unit * off, h * off]).to(ytype)
    norm_case(ops, rows.to(BF16), y, torch.ones(384), 1e-6)


def test_norm_of_special_gains(ops):
    """gains and rows at the ends of what fp32 products can be trusted with"""
    k = 512
    g = torch.Generator().manual_seed(3)
    h = torch.randn(6, k, generator=g) * torch.tensor([1.0, 1e-25, 1e25, 1e-38, 1e37, 1.0])[:, None]
    gain = torch.randn(k, generator=g) * 2.0 ** torch.randint(-140, 120, (k,), generator=g).float()
    gain[::7] = 0.0
    h[:, 3::11] = 0.0
    for eps in (0.0, 1e-6, 1e30):
        norm_case(ops, h, None, gain, eps)
        norm_case(ops, h, None, torch.full((k,), 2.0 ** -140), eps)
        norm_case(ops, h.to(BF16), None, 1 + torch.randn(k, generator=g), eps)


def test_norm_of_special_rows(ops):
    h = torch.randn(8, 640, generator=torch.Generator().manual_seed(1))
    h[0] = 0.0
    h[1] = 1e-30
    h[2] = 1e30                       # its sum of squares passes fp32
    h[3, 100] = float("nan")
    h[4, 7] = float("inf")
    h[5] *= 1e-20
    h[6, :] = 0.0
    h[6, 639] = 5.0
    for dtype in (F32, BF16):
        norm_case(ops, h.to(dtype), None, torch.ones(640), 1e-6)
    gain = torch.ones(640)
    gain[3], gain[4] = 0.0, float("nan")
    norm_case(ops, h[5:].clone(), None, gain, 1e-6)
    norm_case(ops, h[:1].clone(), None, torch.ones(640), 0.0)   # 0 / 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_of_strided_views(ops, dtype):
    big, yb, ob = (activations(6, 1024, s, dtype).cuda() for s in (1, 2, 3))
    for c0, k in ((0, 640), (1, 640), (8, 133)):
        h, y, out = big[:, c0:c0 + k], yb[:, 3:3 + k], ob[:, c0:c0 + k]
        gain = torch.rand(k, device="cuda") + 0.5
        rest = ob.clone()
        want_h, v = ref.norm(h.cpu(), y.cpu(), gain.cpu(), 1e-5)
        rows = ops.scaled_norm(h, gain, 1e-5, y=y, h_out=out)
        assert torch.equal(out.cpu().double(), want_h)
        rest[:, c0:c0 + k] = out
        assert torch.equal(rest, ob)   # nothing beside the view
        same_rows(rows, *ref.quantise(v))


# ---------------------------------------------------------------------------------- products

def product_bound(blocks, mags, dtype):
    if dtype == F32:
        return (blocks + 17) * 2.0 ** -22 * mags, 2.0 ** -24
    return (2.0 ** -10 + blocks * 2.0 ** -20) * mags, 2.0 ** -8


def held(x):
    codes, powers = ref.quantise(x.double())
    return ref.values(codes, powers)


def check_product(out, x, w, k, dtype):
    want, mags = ref.product(held(x), held(w))
    err, half = product_bound(ref.padded(k)[0], mags, dtype)
    got = out.cpu().double()
    bad = (got - want).abs() > err + half * (want.abs() + err)
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / (mags + 1e-300)).max()))
    return float(((got - want).norm() / want.norm().clamp(min=1e-300)))


MATMULS = [(1, 1, 1), (1, 16, 128), (1, 5, 300), (1, 4608, 3584), (2, 100, 1000), (8, 257, 513), (15, 48, 640), (16, 130, 1024), (17, 129, 1100),
           (31, 1001, 1000), (33, 64, 129), (48, 300, 2048), (64, 500, 1500), (65, 16, 4096), (96, 1000, 700), (128, 256, 128), (129, 257, 384),
           (200, 513, 1153), (255, 1024, 896), (256, 768, 512), (257, 300, 3000), (511, 640, 1280), (700, 1100, 300), (1023, 520, 260), (3, 96, 18944), (12, 100, 21800), (16, 60, 40000), (16, 200, 16384), (9, 30, 30000)]
# sizes whose plans have each shape of tile, over all of k and over parts of it
MATMULS += [(1500, 700, 100), (2049, 16, 2000), (65, 20000, 100), (257, 700, 4100), (1500, 1300, 100), (700, 700, 10000), (400, 1000, 4100), (3000, 1300, 100),
            (65, 2000, 10000), (1500, 1300, 2900), (700, 1000, 4100), (1500, 300, 10000), (1500, 1300, 4100)]


@pytest.mark.parametrize("m,n,k", MATMULS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_product(ops, m, n, k, dtype):
    x, w = activations(m, k, m + 3 * n + k), weights(n, k, n + k)
    out = ops.scaled_matmul(ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda()), dtype=dtype)
    off = check_product(out, x, w, k, dtype)
    print(f"  {m} x {n} x {k} {dtype}: {off:.2e} off", flush=True)


@pytest.mark.parametrize("m", [1, 20, 150, 300])
def test_product_writes_its_rows_and_columns_alone(ops, m):
    n, k = 133, 384
    x, w = activations(m, k, 5), weights(n, k, 6)
    for dtype, first, width in ((F32, 4, 160), (F32, 3, 139), (BF16, 1, 140), (BF16, 8, 160)):
        big = torch.full((m + 3, width), -7.0, dtype=dtype, device="cuda")
        out = ops.scaled_matmul(ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda()), out=big[1:m + 1, first:first + n])
        check_product(out, x, w, k, dtype)
        big[1:m + 1, first:first + n] = -7.0
        assert bool((big == -7.0).all())


@pytest.mark.parametrize("m", [1, 9, 40, 130, 300])
def test_product_of_special_rows(ops, m):
    """a row of zeros gives zeros, a NaN its own row alone; large and small powers"""
    n, k = 96, 640
    x, w = activations(m, k, 5), weights(n, k, 6, F32)
    x[m // 2] = 0.0
    x[m - 1] *= 1e30
    w[3] *= 1e-30
    w[5] = 0.0
    if m > 2:
        x[0, 200] = float("nan")
    rows, ww = ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda())
    out = ops.scaled_matmul(rows, ww).cpu()
    if m > 2:
        assert bool(out[0].isnan().all())
        check_product(out[1:], x[1:], w, k, F32)
    else:
        check_product(out, x, w, k, F32)


@pytest.mark.parametrize("m", [1, 16, 40, 200])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_product_of_blocks_of_very_different_sizes(ops, m, dtype):
    """weights whose blocks are 2^-10 to 2^-40 of their row's largest, with inputs that make them matter"""
    n, k = 40, 640
    x, w = activations(m, k, 5, spread=1.0), weights(n, k, 6, F32)
    down = torch.tensor([0.0, 10, 16, 24, 40]).repeat_interleave(128)
    w[:20] *= 2.0 ** -down
    x[::2] *= 2.0 ** (down - 8)
    hx, hw = held(x), held(w)
    want, mags = ref.product(hx, hw)
    err, half = product_bound(5, mags, dtype)
    if dtype == F32:
        top = 2.0 ** (ref.quantise(w.double())[1][:, :5].amax(1).double() - 127)
        err = err + 2.0 ** -25 * top * hx.abs().sum(1, keepdim=True)
    got = ops.scaled_matmul(ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda()), dtype=dtype).cpu().double()
    assert bool(((got - want).abs() <= err + half * (want.abs() + err)).all())


@pytest.mark.parametrize("m", [1, 32, 100, 400])
def test_product_is_the_same_every_time(ops, m):
    x, w = activations(m, 3584, 1).cuda(), weights(512, 3584, 2).cuda()
    rows, ww = ops.scaled_rows(x), ops.ScaledWeights(w)
    first = ops.scaled_matmul(rows, ww)
    for _ in range(5):
        assert torch.equal(ops.scaled_matmul(rows, ww), first)


# ---------------------------------------------------------------------------------- gated

def check_gated(rows, x, wg, wu, n, k):
    hx = held(x)
    (g, gm), (u, um) = ref.product(hx, held(wg)), ref.product(hx, held(wu))
    blocks = ref.padded(k)[0]
    dg, du = product_bound(blocks, gm, F32)[0], product_bound(blocks, um, F32)[0]
    silu = g * torch.sigmoid(g)
    a = silu * u
    err = 1.1 * dg * (u.abs() + du) + silu.abs() * du + 16 * 2.0 ** -24 * a.abs() + 2.0 ** -140
    m = a.shape[0]
    nb, pitch = ref.padded(n)
    assert tuple(rows.codes.shape) == (m, nb * 128) and tuple(rows.scales.shape) == (m, pitch)
    powers = bits(rows.scales)
    least = (a.abs() - err).clamp(min=0)
    low, high = ref.quantise(least)[1], ref.quantise(a.abs() + err)[1]
    # (a block that may be all zeros may have any lower power)
    low[:, :nb][torch.nn.functional.pad(least, (0, nb * 128 - n)).view(m, nb, 128).amax(-1) == 0] = 1
    assert bool((powers[:, nb:] == 127).all()) and bool((bits(rows.codes)[:, n:] == 0).all())
    zero = torch.nn.functional.pad(a, (0, nb * 128 - n)).view(m, nb, 128).abs().amax(-1) == 0
    inside = (powers[:, :nb] >= low[:, :nb]) & (powers[:, :nb] <= high[:, :nb])
    assert bool((inside | zero).all())
    scale = (2.0 ** (powers[:, :nb].double() - 127)).repeat_interleave(128, 1)[:, :n]
    got = ref.values(rows.codes, rows.scales)[:, :n]
    lo, hi = (ref.TABLE[ref.nearest(((a.abs() + s * err) / scale).clamp(0, 448)).long()] for s in (-1, 1))
    mag = got.abs() / scale
    near_zero = a.abs() <= err
    if a.numel() >= 1000:
        want = ref.values(*ref.quantise(a))[:, :n]
        assert float((got != want).double().mean()) <= 0.001
    assert bool(((mag >= lo) & (mag <= hi)).all()), int(((mag < lo) | (mag > hi)).sum())
    assert bool(((got * a >= 0) | near_zero).all())


GATED = [(1, 1, 1), (1, 128, 128), (1, 200, 1000), (1, 1000, 3584), (7, 129, 500), (16, 256, 512), (17, 384, 1030), (32, 100, 640), (33, 640, 300),
         (64, 130, 1024), (65, 512, 520), (100, 300, 2000), (128, 1024, 256), (130, 700, 384), (256, 256, 128), (300, 900, 640), (513, 130, 1100)]
GATED += [(17, 16, 1500), (4099, 16, 100), (700, 16, 2900), (3000, 300, 100), (2049, 16, 2000), (1500, 1300, 100), (4099, 16, 2000)]   # (as above)


@pytest.mark.parametrize("m,n,k", GATED)
def test_gated(ops, m, n, k):
    x, wg, wu = activations(m, k, m + n + k, spread=5.0), weights(n, k, n), weights(n, k, n + 1)
    rows = ops.scaled_gated(ops.scaled_rows(x.cuda()), ops.ScaledWeights(wg.cuda(), wu.cuda()))
    check_gated(rows, x, wg, wu, n, k)


@pytest.mark.parametrize("m", [1, 40, 140])
def test_gated_of_special_rows(ops, m):
    n, k = 200, 384
    x, wg, wu = activations(m, k, 3), weights(n, k, 4, F32), weights(n, k, 5, F32)
    wg[0] *= 1e4        # silu saturated on both sides
    wu[1] = 0.0
    x[m // 2] = 0.0
    rows = ops.scaled_gated(ops.scaled_rows(x.cuda()), ops.ScaledWeights(wg.cuda(), wu.cuda()))
    check_gated(rows, x, wg, wu, n, k)
    if m > 2:
        x[1, 0] = float("inf")
        rows = ops.scaled_gated(ops.scaled_rows(x.cuda()), ops.ScaledWeights(wg.cuda(), wu.cuda()))
        codes = bits(rows.codes)
        assert bool(((codes[1, :n] & 127) == 127).all()) and bool((bits(rows.scales)[1] == 127).all())
        assert not bool(((torch.cat([codes[:1], codes[2:]]) & 127) == 127).any())


# ---------------------------------------------------------------------------------- together, and how they are called

def test_a_layer_of_them_together(ops):
    """norm, product, rows, product, norm with the residual, gated, product: each stage against 64 bits on the stage's
    own input, on a stream that is not the current device's default, all enqueued before anything is looked at"""
    m, d, F = 37, 640, 1100
    h, gain = activations(m, d, 1), 1 + 0.1 * torch.randn(d, generator=torch.Generator().manual_seed(2))
    wa, wo, wg, wu, wd = (weights(*s, seed=i) for i, s in enumerate([(d + 128, d), (d, d + 128), (F, d), (F, d), (d, F)]))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        hd = h.cuda()
        x1 = ops.scaled_norm(hd, gain.cuda(), 1e-6)
        q = ops.scaled_matmul(x1, ops.ScaledWeights(wa.cuda()))
        x2 = ops.scaled_rows(q)
        o = ops.scaled_matmul(x2, ops.ScaledWeights(wo.cuda()))
        x3 = ops.scaled_norm(hd, gain.cuda(), 1e-6, y=o)
        x4 = ops.scaled_gated(x3, ops.ScaledWeights(wg.cuda(), wu.cuda()))
        y = ops.scaled_matmul(x4, ops.ScaledWeights(wd.cuda()))
    stream.synchronize()
    same_rows(x1, *ref.quantise(ref.norm(h, None, gain, 1e-6)[1]))
    v1 = ref.values(x1.codes, x1.scales)[:, :d]
    check_product(q, v1, wa, d, F32)
    same_rows(x2, *ref.quantise(q.cpu().double()))
    check_product(o, q.cpu(), wo, d + 128, F32)
    want_h, v = ref.norm(h, o.cpu(), gain, 1e-6)
    assert torch.equal(hd.cpu().double(), want_h)
    same_rows(x3, *ref.quantise(v))
    v3 = ref.values(x3.codes, x3.scales)[:, :d]
    check_gated(x4, v3, wg, wu, F, d)
    check_product(y, ref.values(x4.codes, x4.scales)[:, :F], wd, F, F32)


@pytest.mark.parametrize("m", [1, 24, 200])
def test_captured_and_replayed(ops, m):
    """all four in a captured graph: every replay equals the eager results, with eager work on the same weights and new
    inputs between the replays"""
    d, F = 512, 700
    gain = torch.ones(d, device="cuda")
    w, pair = ops.ScaledWeights(weights(384, d, 1).cuda()), ops.ScaledWeights(weights(F, d, 2).cuda(), weights(F, d, 3).cuda())
    h, y = activations(m, d, 1).cuda(), activations(m, d, 2).cuda()
    h_out, rows, act = torch.empty_like(h), ops.ScaledRows.empty(m, d), ops.ScaledRows.empty(m, F)
    back, out = ops.ScaledRows.empty(m, 384), torch.empty(m, 384, device="cuda")

    def step():
        ops.scaled_norm(h, gain, 1e-6, y=y, h_out=h_out, out=rows)
        ops.scaled_matmul(rows, w, out=out)
        ops.scaled_rows(out, out=back)
        ops.scaled_gated(rows, pair, out=act)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        h.copy_(activations(m, d, 10 + turn))
        y.copy_(activations(m, d, 20 + turn))
        for t in (h_out, out, rows.codes.view(torch.uint8), act.codes.view(torch.uint8), back.codes.view(torch.uint8)):
            t.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (h_out, out, bits(rows.codes), bits(act.codes), bits(act.scales), bits(back.codes), bits(back.scales))]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (h_out, out, bits(rows.codes), bits(act.codes), bits(act.scales), bits(back.codes), bits(back.scales))):
            assert torch.equal(a, b)


def test_more_rows_than_a_launch_takes(ops):
    """2^27 + 3 rows, whose codes pass 32 bits and whose launches are cut: the same as of 2^22 rows at a time"""
    m, piece = (1 << 27) + 3, 1 << 22
    x = torch.randn(m, 1, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    w, pair = ops.ScaledWeights(weights(2, 1, 1).cuda()), ops.ScaledWeights(weights(2, 1, 2).cuda() * 50, weights(2, 1, 3).cuda())
    rows = ops.scaled_rows(x)
    out, act = ops.scaled_matmul(rows, w, dtype=BF16), ops.scaled_gated(rows, pair)
    for r in range(0, m, piece):
        part = ops.scaled_rows(x[r:r + piece])
        act_part = ops.scaled_gated(part, pair)
        for whole, cut in ((rows, part), (act, act_part)):
            for a, b in ((whole.codes, cut.codes), (whole.scales, cut.scales)):
                assert torch.equal(a.view(torch.uint8)[r:r + piece], b.view(torch.uint8)), r
        assert torch.equal(out[r:r + piece], ops.scaled_matmul(part, w, dtype=BF16)), r


def test_norm_of_more_rows_than_a_launch_takes(ops):
    m, k, piece = (1 << 21) + 5, 40, 1 << 19
    h, y = (torch.randn(m, k, device="cuda", generator=torch.Generator("cuda").manual_seed(s)).bfloat16() for s in (1, 2))
    gain, out = torch.ones(k, device="cuda"), torch.empty_like(h)
    rows = ops.scaled_norm(h, gain, 1e-6, y=y, h_out=out)
    for r in range(0, m, piece):
        o = torch.empty_like(h[r:r + piece])
        part = ops.scaled_norm(h[r:r + piece], gain, 1e-6, y=y[r:r + piece], h_out=o)
        assert torch.equal(o, out[r:r + piece]), r
        for a, b in ((rows.codes, part.codes), (rows.scales, part.scales)):
            assert torch.equal(a.view(torch.uint8)[r:r + piece], b.view(torch.uint8)), r


def test_no_rows(ops):
    w, pair = ops.ScaledWeights(weights(20, 64, 1).cuda()), ops.ScaledWeights(weights(20, 64, 2).cuda(), weights(20, 64, 3).cuda())
    x = torch.empty(0, 64, device="cuda")
    rows = ops.scaled_rows(x)
    assert rows.m == 0 and ops.scaled_norm(x, torch.ones(64, device="cuda"), 1e-6, y=x.clone()).m == 0
    assert tuple(ops.scaled_matmul(rows, w).shape) == (0, 20) and ops.scaled_gated(rows, pair).m == 0


def test_two_calls_at_once(ops):
    """two streams with one set of weights, each with its own workspace"""
    m, n, k = 150, 256, 2048
    w = ops.ScaledWeights(weights(n, k, 1).cuda())
    xs = [ops.scaled_rows(activations(m, k, s).cuda()) for s in (1, 2)]
    want = [ops.scaled_matmul(x, w) for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ops.scaled_matmul(xs[i], w))
    torch.cuda.synchronize()
    for i in (0, 1):
        for t in got[i]:
            assert torch.equal(t, want[i])


def test_values_and_refusals(ops):
    from paper_2603_09215_amd import SparkError
    x = activations(5, 300, 1).cuda()
    rows = ops.scaled_rows(x)
    assert torch.equal(rows.values().cpu().double(), ref.values(*ref.quantise(x.cpu().double()))[:, :300])
    w = ops.ScaledWeights(weights(40, 300, 1).cuda())
    pair = ops.ScaledWeights(weights(40, 300, 1).cuda(), weights(40, 300, 2).cuda())
    square = ops.ScaledWeights(weights(300, 300, 1).cuda(), weights(300, 300, 2).cuda())
    gain = torch.ones(300, device="cuda")
    short = ops.ScaledRows.empty(5, 200)
    for call in (lambda: ops.scaled_rows(x.cpu()), lambda: ops.scaled_rows(x.half()), lambda: ops.scaled_rows(x[0]), lambda: ops.scaled_rows(x.t()),
                 lambda: ops.scaled_rows(x, out=short), lambda: ops.scaled_rows(x[:1].expand(5, 300)),
                 lambda: ops.scaled_norm(x, gain[:299], 1e-6), lambda: ops.scaled_norm(x, gain, -1.0), lambda: ops.scaled_norm(x, gain.double(), 1e-6),
                 lambda: ops.scaled_norm(x, gain, 1e-6, y=x[:4]), lambda: ops.scaled_norm(x, gain, 1e-6, h_out=x.bfloat16()),
                 lambda: ops.scaled_norm(x, gain, float("nan")),
                 lambda: ops.scaled_matmul(rows, pair), lambda: ops.scaled_matmul(short, w), lambda: ops.scaled_matmul(rows, w, dtype=torch.float16),
                 lambda: ops.scaled_matmul(rows, w, out=torch.empty(5, 41, device="cuda")), lambda: ops.scaled_gated(rows, w),
                 lambda: ops.scaled_gated(rows, pair, out=short), lambda: ops.scaled_gated(rows, square, out=rows), lambda: ops.ScaledWeights(x.double()),
                 lambda: ops.ScaledWeights(x, x[:4]), lambda: ops.ScaledRows(rows.codes, rows.scales, 600)):
        with pytest.raises(SparkError):
            call()
