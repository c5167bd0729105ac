"""Microscaled rows and weights, RMSNorm into them and the product on them (GPU only), against mx_reference.

Quantisation is exact, so its bytes are equal to the reference's.  Where a computed value is quantised (SiLU, RMSNorm) it is off by
up to FP32 * |y| (a dozen fp32 roundings and functions of 2 ulp, 2^-24 each), and the code may be a neighbour where y lies on
a border: then the value that the code stands for is within half a step of the format and that error.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import mx_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
FP32 = 64 * 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_01699_amd import binding
    return binding


TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def up(n, m):
    return -(-n // m) * m


def buffers(rows, K, bits):
    """codes and scales, with bytes that have to go"""
    return (torch.full((rows, up(K, 128) * bits // 8), 0xAB, dtype=torch.uint8, device="cuda"),
            torch.full((rows, up(K, 128) // 32), 0xAB, dtype=torch.uint8, device="cuda"))


def codes_of(codes, bits):
    c = codes.cpu().numpy()
    return c if bits == 8 else R.unpair(c)


def data(rows, K, dtype, seed=0, wide=True):
    """rows whose blocks' magnitudes differ by many powers of two"""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, K, generator=g)
    if wide:
        x *= 2.0 ** torch.randint(-30, 30, (rows, up(K, 32) // 32), generator=g).repeat_interleave(32, 1)[:, :K]
    return x.to(TYPES[dtype])


def special(dtype):
    """blocks of zeros, of the type's smallest and largest values, of ties, of infinities and NaN, and borders of the scale"""
    t = TYPES[dtype]
    tiny = 2.0 ** -149 if dtype == "fp32" else 2.0 ** -133
    big = float(torch.finfo(t).max)
    rows = []
    rows.append(torch.zeros(128)); rows[-1][3] = -0.0
    rows.append(torch.arange(128) % 7 * tiny)
    rows.append(torch.full((128,), 2.0 ** -126) * torch.linspace(-1, 1, 128))
    rows.append(torch.linspace(-1, 1, 128) * big)
    for base in (448.0, 6.0, 447.9, 6.1, 449.0, 464.0, 480.0):
        r = torch.linspace(-1, 1, 128, dtype=torch.float64) * base
        r[::32] = base
        rows.append(r)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, 1.0] + [1 + (2 * i + 1) / 16 for i in range(8)] + [(2 * i + 1) / 1024 for i in range(13)] + [448.0])
    rows += [torch.cat((ties, -ties, ties, -ties)), torch.cat((ties[:8], -ties[:8])).repeat(8)]
    for i, v in enumerate((float("inf"), -float("inf"), float("nan"))):
        r = torch.linspace(-3, 3, 128)
        r[5 + 40 * i] = v
        rows.append(r)
    rows.append(torch.full((128,), float("nan")))
    return torch.stack([r.double() for r in rows]).to(t)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
def test_special_values_to_the_byte(B, bits, dtype):
    x = special(dtype)
    codes, scales = buffers(*x.shape, bits)
    B.sjd_mx_quantize(bits, x.cuda(), codes, scales)
    want, ws = R.quantise(x.double().numpy(), bits)
    assert np.array_equal(scales.cpu().numpy(), ws)
    assert np.array_equal(codes_of(codes, bits), want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 31), (2, 32), (5, 33), (17, 127), (4, 128), (3, 129), (130, 257), (7, 1536), (2, 11008), (1000, 40)])
def test_quantise_to_the_byte(B, rows, K, bits, dtype):
    x = data(rows, K, dtype)
    codes, scales = buffers(rows, K, bits)
    B.sjd_mx_quantize(bits, x.cuda(), codes, scales)
    want, ws = R.quantise(x.double().numpy(), bits)
    assert np.array_equal(scales.cpu().numpy(), ws)
    assert np.array_equal(codes_of(codes, bits), want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("off,pad", [(0, 8), (8, 0), (1, 5), (3, 0)])
def test_rows_of_a_wider_matrix_at_any_address(B, off, pad, dtype):
    """off, pad: columns in front of and behind the rows; odd ones leave the rows unaligned"""
    wide = data(9, off + 200 + pad, dtype, wide=False).cuda()
    x = wide[:, off:off + 200]
    codes, scales = buffers(9, 200, 8)
    B.sjd_mx_quantize(8, x, codes, scales)
    want, ws = R.quantise(x.double().cpu().numpy(), 8)
    assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(codes_of(codes, 8), want)


def near(y, codes, scales, bits):
    """codes and scales hold y (64 bits), which the kernel knew to FP32 * |y|: see above"""
    rows, K = y.shape
    Kp = up(K, 128)
    p = np.zeros((rows, Kp))
    p[:, :K] = y
    s = 2.0 ** (scales.astype(np.float64) - 127)
    amax = np.abs(p).reshape(rows, -1, 32).max(-1)
    lo, hi = (R.scale_bytes(np.float32(amax * (1 + f)).astype(np.float64), bits) for f in (-FP32, FP32))
    assert ((scales >= lo) & (scales <= hi)).all()
    got = R.values(codes, scales, bits)
    s = np.repeat(s, 32, axis=-1)
    # (half a step just above a power of two is twice the one below it)
    room = np.abs(p) * FP32 + 0.5 * s * np.maximum(R.step(p / s * (1 + FP32), bits), R.step(p / s, bits)) + 2.0 ** -149
    assert (np.abs(got - p) <= room).all(), np.max(np.abs(got - p) / room)
    assert (codes[:, K:] & (127 if bits == 8 else 7) == 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,F", [(1, 64), (3, 100), (33, 4096)])
def test_swiglu(B, rows, F, bits, dtype):
    h = (3 * data(rows, 2 * F, dtype, seed=2, wide=False).float()).to(TYPES[dtype])
    h[0, 0], h[0, 1] = -200.0, 200.0                                   # exp overflows, and vanishes
    h = h.cuda()
    codes, scales = buffers(rows, F, bits)
    B.sjd_mx_quantize(bits, h[:, :F], codes, scales, up=h[:, F:])
    h = h.double().cpu().numpy()
    with np.errstate(over="ignore"):
        y = h[:, :F] / (1 + np.exp(-h[:, :F])) * h[:, F:]
    y[np.abs(y) < 1e-30] = 0                                           # (fp32 gives -0 for -200 / (1 + inf))
    near(y, codes_of(codes, bits), scales.cpu().numpy(), bits)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,d,pad", [(1, 1, 0), (2, 33, 0), (3, 128, 4), (5, 1536, 0), (4, 1537, 3), (2, 4096, 0), (1, 8192, 0), (2, 8200, 0), (1, 20001, 0)])
def test_rmsnorm(B, rows, d, pad, bits, dtype):
    x, res = data(rows, d, dtype, seed=3, wide=False).cuda(), data(rows, d + pad, "fp32", seed=4, wide=False).cuda()
    gain = 1 + 0.1 * torch.randn(d, generator=torch.Generator().manual_seed(5)).cuda()
    if rows > 1:
        x[1], res[1] = 0, 0                                            # a row of zeros stays one
    before, r = res.clone(), res[:, :d]
    codes, scales = buffers(rows, d, bits)
    B.sjd_mx_rmsnorm(bits, x, r, gain, 1e-5, codes, scales)
    h = before[:, :d] + x.float()                                      # one fp32 addition
    assert torch.equal(r, h) and torch.equal(res[:, d:], before[:, d:])
    h = h.double().cpu().numpy()
    y = h / np.sqrt((h * h).mean(-1, keepdims=True) + 1e-5) * gain.double().cpu().numpy()
    near(y, codes_of(codes, bits), scales.cpu().numpy(), bits)


@pytest.mark.parametrize("which", ["x", "resid"])
def test_rmsnorm_of_one_input(B, which):
    h = data(7, 1000, "fp32", seed=6, wide=False).cuda()
    keep, gain = h.clone(), torch.ones(1000, device="cuda")
    codes, scales = buffers(7, 1000, 8)
    B.sjd_mx_rmsnorm(8, h if which == "x" else None, h if which == "resid" else None, gain, 0.0, codes, scales)
    assert torch.equal(h, keep)
    y = h.double().cpu().numpy()
    near(y / np.sqrt((y * y).mean(-1, keepdims=True)), codes_of(codes, 8), scales.cpu().numpy(), 8)


def test_rmsnorm_keeps_a_bad_row_to_itself(B):
    x = data(4, 256, "fp32", seed=7, wide=False).cuda()
    gain = torch.ones(256, device="cuda")
    a, b = buffers(4, 256, 8), buffers(4, 256, 8)
    B.sjd_mx_rmsnorm(8, x, None, gain, 1e-5, *a)
    x[1, 5], x[2, 40] = float("nan"), float("inf")
    B.sjd_mx_rmsnorm(8, x, None, gain, 1e-5, *b)
    for r in (0, 3):
        assert torch.equal(a[0][r], b[0][r]) and torch.equal(a[1][r], b[1][r])
    assert (b[0][1] == 0x7F).all()                                     # the sum is NaN
    assert b[0][2, 40] == 0x7F and (b[0][2].cpu().numpy() & 127)[np.arange(256) != 40].max() == 0      # 1 / inf


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,K", [(1, 1), (5, 33), (16, 512), (17, 513), (40, 1536), (33, 1300)])
def test_weights_to_the_byte(B, N, K, dtype):
    w = data(N, K, dtype, seed=8)
    if N > 2:
        w[2, 0] = float("nan")
    packed = torch.full((B.sjd_mx_weights_bytes(N, K),), 0xAB, dtype=torch.uint8, device="cuda")
    B.sjd_mx_weights(w.cuda(), packed)
    assert np.array_equal(packed.cpu().numpy(), R.pack_weights(*R.quantise(w.double().numpy(), 4), N, K))


def operands(M, N, K, bits, seed=9):
    """(codes, scales, packed) on the GPU and the values they stand for"""
    a, w = data(M, K, "fp32", seed, wide=False).numpy(), 0.02 * data(N, K, "fp32", seed + 1, wide=False).numpy()
    a *= 2.0 ** np.random.RandomState(seed).randint(-3, 4, (M, 1))
    ca, sa = R.quantise(a, bits)
    cw, sw = R.quantise(w, 4)
    gpu = [torch.from_numpy(x).cuda() for x in (ca if bits == 8 else R.pair(ca), sa, R.pack_weights(cw, sw, N, K))]
    return gpu, R.values(ca, sa, bits), R.values(cw, sw, 4)


def product(B, gpu, M, N, K, bits, dtype, out=None):
    out = torch.full((M, N), float("nan"), dtype=TYPES[dtype], device="cuda") if out is None else out
    need = B.sjd_mx_product_workspace(M, N, K)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    B.sjd_mx_product(bits, *gpu, K, out, ws)
    return out


def check_product(out, a, w, K, dtype):
    """Products are exact; a sum of K of them in fp32, in any order, is off by at most K 2^-24 sum |a w| (K / 2 on
    average would be its square root: the 2-norm is held to 1e-6); bf16 rounds once, by 2^-8 of the value"""
    want, mag = a @ w.T, np.abs(a) @ np.abs(w).T
    got = out.double().cpu().numpy()
    half = 2.0 ** -8 if dtype == "bf16" else 0
    room = K * 2.0 ** -24 * mag * (1 + half) + half * np.abs(want) + 2.0 ** -149
    assert (np.abs(got - want) <= room).all(), np.max(np.abs(got - want) / room)
    if dtype == "fp32":
        assert np.linalg.norm(got - want) <= 1e-6 * np.linalg.norm(want) + 1e-30


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 128, 129, 200, 257])
@pytest.mark.parametrize("N,K", [(1, 1), (17, 130), (100, 640), (260, 1536), (48, 4096)])
def test_product(B, M, N, K, bits, dtype):
    gpu, a, w = operands(M, N, K, bits)
    check_product(product(B, gpu, M, N, K, bits, dtype), a, w, K, dtype)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (16, 4608, 1536), (33, 1536, 4096), (128, 4096, 1024), (300, 1100, 700), (513, 2048, 256), (1, 9000, 11008)])
def test_product_of_larger_sizes(B, M, N, K, bits):
    gpu, a, w = operands(M, N, K, bits)
    check_product(product(B, gpu, M, N, K, bits, "fp32"), a, w, K, "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [1, 20, 70, 300])
@pytest.mark.parametrize("N,pad", [(50, 6), (64, 64), (37, 0)])
def test_product_into_rows_of_a_wider_matrix(B, M, N, pad, dtype):
    gpu, a, w = operands(M, N, 256, 8)
    wide = torch.full((M, N + pad), 7.0, dtype=TYPES[dtype], device="cuda")
    check_product(product(B, gpu, M, N, 256, 8, dtype, wide[:, :N]), a, w, 256, dtype)
    assert (wide[:, N:] == 7).all()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M", [3, 40, 140, 300])
def test_nan_stays_in_its_row_and_column(B, M, bits):
    N, K = 96, 1024
    gpu, a, w = operands(M, N, K, bits)
    ref = product(B, gpu, M, N, K, bits, "fp32")
    codes, scales, packed = (t.clone() for t in gpu)
    if bits == 8:
        codes[1, 700] = 0x7F
    else:
        scales[1, 20] = 255
    packed.view(6, 2, 4352)[3, 1, 4096 + 4 * (16 * 2 + 5) + 1] = 255       # feature 53, a block of the second 512 values
    out = product(B, (codes, scales, packed), M, N, K, bits, "fp32")
    hit = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    hit[1], hit[:, 53] = True, True
    assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], ref[~hit])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [2, 20, 70, 300])
@pytest.mark.parametrize("K", [100, 130, 640, 1500])
def test_nan_blocks_of_a_row_leave_the_row_before_alone(B, K, M, dtype):
    """K that ends inside a record of 512 values: what is read behind a row is the next row's"""
    N = 96
    gpu, a, w = operands(M, N, K, 4)
    ref = product(B, gpu, M, N, K, 4, dtype)
    scales = gpu[1].clone()
    scales[1::2] = 255
    out = product(B, (gpu[0], scales, gpu[2]), M, N, K, 4, dtype)
    assert torch.isnan(out[1::2]).all() and torch.equal(out[::2], ref[::2])


@pytest.mark.parametrize("M", [1, 16, 50, 200])
def test_calls_agree_and_are_captured(B, M):
    """the same bits on another stream, and from replays of a graph with eager work between them"""
    N, K = 1536, 1536
    gpu, a, w = operands(M, N, K, 8)
    ref = product(B, gpu, M, N, K, 8, "fp32")
    x, r = data(M, K, "fp32", seed=12, wide=False).cuda(), torch.zeros(M, K, device="cuda")
    gain = torch.ones(K, device="cuda")
    codes, scales = buffers(M, K, 8)
    out = torch.empty_like(ref)
    ws = torch.empty(B.sjd_mx_product_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.sjd_mx_product(8, *gpu, K, out, ws, stream=side)
    side.synchronize()
    assert torch.equal(out, ref)
    B.sjd_mx_rmsnorm(8, x, None, gain, 1e-5, codes, scales)
    B.sjd_mx_product(8, codes, scales, gpu[2], K, out, ws)
    want = out.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream()
        B.sjd_mx_rmsnorm(8, x, r, gain, 1e-5, codes, scales, stream=s)
        B.sjd_mx_product(8, codes, scales, gpu[2], K, out, ws, stream=s)
    for _ in range(4):
        r.zero_(); out.fill_(float("nan")); codes.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(r, x)


def test_matrices_of_more_than_4_gib(B):
    """what lies behind 2^31 elements and 2^32 bytes: the last rows give what they give alone"""
    K, dev = 1 << 16, "cuda"
    x = torch.empty(33000, K, dtype=torch.bfloat16, device=dev)
    x.view(torch.int16).random_(-0x3FFF, 0x3FFF)                       # (any finite bits below 2)
    tail = x[-32:].contiguous()
    codes, scales = buffers(*x.shape, 8)
    few = buffers(32, K, 8)
    B.sjd_mx_quantize(8, x, codes, scales)
    B.sjd_mx_quantize(8, tail, *few)
    assert torch.equal(codes[-32:], few[0]) and torch.equal(scales[-32:], few[1])
    codes.zero_()
    gain = torch.ones(K, device=dev)
    B.sjd_mx_rmsnorm(8, x, None, gain, 1e-5, codes, scales)
    B.sjd_mx_rmsnorm(8, tail, None, gain, 1e-5, *few)
    assert torch.equal(codes[-32:], few[0]) and torch.equal(scales[-32:], few[1])
    del codes, scales
    packed, part = (torch.empty(B.sjd_mx_weights_bytes(n, K), dtype=torch.uint8, device=dev) for n in (33000, 24))
    B.sjd_mx_weights(x, packed)
    B.sjd_mx_weights(x[-24:], part)                                    # 33000 = 16 * 2061 + 24: whole tiles
    assert torch.equal(packed[-part.numel():], part)


@pytest.mark.parametrize("M,N,K,dtype", [(70000, 16390, 128, "fp32"), (2200000, 20, 200, "fp32"), (3, 2200000, 100, "fp32")])
def test_products_of_very_many_rows_or_features(B, M, N, K, dtype):
    """outputs of more than 4 GiB, more rows than a grid's second dimension holds; the last rows and features against the reference"""
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = torch.randn(M, K, device="cuda", generator=g), torch.randn(N, K, device="cuda", generator=g)
    codes, scales = buffers(M, K, 8)
    packed = torch.empty(B.sjd_mx_weights_bytes(N, K), dtype=torch.uint8, device="cuda")
    B.sjd_mx_quantize(8, x, codes, scales)
    B.sjd_mx_weights(w, packed)
    out = product(B, (codes, scales, packed), M, N, K, 8, dtype)
    rows, cols = min(M, 40), min(N, 50)
    a = R.values(codes[-rows:].cpu().numpy(), scales[-rows:].cpu().numpy(), 8)
    v = R.values(*R.quantise(w[-cols:].cpu().double().numpy(), 4), 4)
    check_product(out[-rows:, -cols:], a, v, K, dtype)


def test_products_at_the_same_time(B):
    """two streams, a workspace each, and a size that is split over K (so that both use theirs)"""
    M, N, K = 128, 4096, 11008
    assert B.sjd_mx_product_workspace(M, N, K) > 0
    gpu = [operands(M, N, K, 8, seed=20 + i)[0] for i in range(2)]
    ref = [product(B, x, M, N, K, 8, "fp32") for x in gpu]
    outs, ws = [torch.zeros_like(r) for r in ref], [torch.empty(B.sjd_mx_product_workspace(M, N, K), dtype=torch.uint8, device="cuda") for _ in gpu]
    streams = [torch.cuda.Stream() for _ in gpu]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, o, w, s in zip(gpu, outs, ws, streams):
            B.sjd_mx_product(8, *x, K, o, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, r) for o, r in zip(outs, ref))


def test_the_binding_refuses(B):
    """sizes, types and layouts that do not fit each other"""
    def e(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def u8(*shape):
        return e(*shape, dtype=torch.uint8)

    x, c, s, p, o = e(4, 64), u8(4, 128), u8(4, 4), u8(4352), e(4, 16)
    cache, cs, n = u8(2, 1, 2, 64 * 64), u8(2, 1, 2, 2), torch.zeros(2, dtype=torch.int32, device="cuda")
    bad = [lambda: B.sjd_mx_quantize(8, x, u8(4, 64), s), lambda: B.sjd_mx_quantize(8, x, c, u8(4, 2)), lambda: B.sjd_mx_quantize(5, x, c, s),
           lambda: B.sjd_mx_quantize(8, x.half(), c, s), lambda: B.sjd_mx_quantize(8, x.t(), u8(64, 128), u8(64, 4)), lambda: B.sjd_mx_quantize(8, x[0], c, s),
           lambda: B.sjd_mx_quantize(8, x, c.cpu(), s), lambda: B.sjd_mx_quantize(8, x, c.view(torch.int8), s), lambda: B.sjd_mx_quantize(8, x, c, s, up=x[:, :32]),
           lambda: B.sjd_mx_quantize(8, x, c, s, up=x.bfloat16()), lambda: B.sjd_mx_quantize(8, x, c, s, up=e(4, 128)[:, :64]),
           lambda: B.sjd_mx_quantize(8, x[:1].expand(4, 64), c, s), lambda: B.sjd_mx_quantize(8, x, u8(4, 256)[:, ::2], s),
           lambda: B.sjd_mx_rmsnorm(8, x, x.bfloat16(), e(64), 1e-5, c, s), lambda: B.sjd_mx_rmsnorm(8, x, None, e(63), 1e-5, c, s),
           lambda: B.sjd_mx_rmsnorm(8, x, e(3, 64), e(64), 1e-5, c, s), lambda: B.sjd_mx_rmsnorm(8, x, None, e(64), -1.0, c, s),
           lambda: B.sjd_mx_weights(x, u8(4353)), lambda: B.sjd_mx_weights(x, u8(4336)),
           lambda: B.sjd_mx_product(8, c, s, p, 129, o, None), lambda: B.sjd_mx_product(8, c, s, p, 64, e(4, 17), None), lambda: B.sjd_mx_product(4, c, s, p, 64, o, None),
           lambda: B.sjd_mx_product(8, c, s, p, 64, e(5, 16), None), lambda: B.sjd_mx_product(8, u8(4 * 128 + 8)[8:].view(4, 128), s, p, 64, o, None),
           lambda: B.sjd_kv8_append(e(4, 64), e(4, 64), n, 1, 1, 64, 64, cache, cs), lambda: B.sjd_kv8_append(e(2, 64), e(2, 64), n.long(), 1, 1, 64, 64, cache, cs),
           lambda: B.sjd_kv8_append(e(2, 64), e(2, 64), n, 1, 1, 64, 65, cache, cs), lambda: B.sjd_kv8_append(e(2, 64), e(2, 65)[:, :64], n, 1, 1, 64, 64, cache, cs),
           lambda: B.sjd_kv8_append(e(2, 64), e(2, 64), n[:0], 1, 1, 64, 64, cache, cs),
           lambda: B.sjd_kv8_attention(e(2, 64), cache, cs, n, 1, 1, 1, 64, 64, 0, 0, e(2, 64, dtype=torch.bfloat16), None),
           lambda: B.sjd_kv8_attention(e(2, 64), cache, cs, n, 1, 1, 1, 64, 64, -1, 0, e(2, 64), None),
           lambda: B.sjd_kv8_attention(e(2, 64), cache, cs[:1], n, 1, 1, 1, 64, 64, 0, 0, e(2, 64), None),
           lambda: B.sjd_kv8_attention(e(2, 64), u8(2, 1, 64, 64 * 64), u8(2, 1, 64, 2), n, 1, 1, 1, 64, 2048, 0, 0, e(2, 64), u8(64))]
    for i, f in enumerate(bad):
        with pytest.raises(B.SjdError) as err:
            f()
        assert err.value.code == B.SJD_EINVAL, i


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
def test_swiglu_of_gates_far_below_zero(B, bits, dtype):
    """e^x below what fp32 holds, times values that bring it back: bf16 and fp32 hold the product"""
    rows, F = 4, 256
    r = np.random.RandomState(15)
    gate = -np.linspace(60, 170, rows * F).reshape(rows, F)
    y = np.exp2(r.randint(-60, 40, (rows, F // 32)).repeat(32, 1)) * (1 + r.rand(rows, F))       # the product's magnitude, much the same in a block
    up = np.sign(r.randn(rows, F)) * np.clip(y / np.abs(gate) * np.exp(-gate), 1e-30, 1e38)
    h = torch.from_numpy(np.concatenate((gate, up), 1)).to(TYPES[dtype]).cuda()
    codes, scales = buffers(rows, F, bits)
    B.sjd_mx_quantize(bits, h[:, :F], codes, scales, up=h[:, F:])
    h = h.double().cpu().numpy()
    near(h[:, :F] / (1 + np.exp(-h[:, :F])) * h[:, F:], codes_of(codes, bits), scales.cpu().numpy(), bits)
