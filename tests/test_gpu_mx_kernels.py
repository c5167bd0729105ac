"""The 4-bit product on each of its kernels (GPU only), whatever the plan would take at these sizes; and products whose sums fp32 holds exactly."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import mx_reference as R  # noqa: E402
from test_gpu_mx import B, TYPES, check_product, operands  # noqa: E402,F401

pytestmark = pytest.mark.gpu

TILES = [(64, 64), (64, 128), (64, 192), (128, 128), (128, 192), (128, 256), (256, 256)]
ROWS = [(16, 16 * t) for t in (1, 2, 3, 4, 6)] + [(32, 16 * t) for t in (1, 2, 3, 4)]
# K of 1 to 9 steps of 128 values and a few more: the loop of four and what is left of it, records that end after 1 to 4 steps, rows
# that end inside a step
LENGTHS = [70, 256, 300, 512, 600, 768, 900, 1024, 1100, 1536, 1900]


def run(B, plan, gpu, M, N, K, bits, dtype, out=None):
    out = torch.full((M, N), float("nan"), dtype=TYPES[dtype], device="cuda") if out is None else out
    ws = torch.full((plan[2] * M * ((N + 3) // 4 * 4) * 4,), 0xFF, dtype=torch.uint8, device="cuda") if plan[2] > 1 else None
    B.sjd_mx_product_test(plan, bits, *gpu, K, out, ws)
    return out


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,cols", ROWS + TILES, ids=lambda v: str(v))
def test_every_kernel(B, rows, cols, bits, dtype):
    """fewer rows than a workgroup has and one more than two have; features that end inside a tile of 16, inside a wave's tiles, and behind them"""
    for i, K in enumerate(LENGTHS):
        M, N = [(rows + 1 if rows > 32 else rows, cols - 3), (2 * rows + 1, cols + 17), (max(rows - 31, 33), 2 * cols + 50), (rows + 16, 31)][i % 4]
        M = max(1, rows - i) if rows == 16 else M
        gpu, a, w = operands(M, N, K, bits, seed=30 + i)
        check_product(run(B, (rows, cols, 1), gpu, M, N, K, bits, dtype), a, w, K, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,cols", TILES, ids=lambda v: str(v))
def test_every_tile_in_slices(B, rows, cols, bits, dtype):
    """K in 2 and 4 slices, the last one shorter, joined by the second kernel; rows of odd length, which it writes value by value"""
    for M, N, K, slices in ((rows + 9, cols + 3, 1100, 2), (77, cols - 1, 2050, 4), (2 * rows, cols + 20, 4096, 2), (70, 50, 5700, 4)):
        gpu, a, w = operands(M, N, K, bits, seed=50 + slices)
        check_product(run(B, (rows, cols, slices), gpu, M, N, K, bits, dtype), a, w, K, dtype)
    wide = torch.full((40, 90), 7.0, dtype=TYPES[dtype], device="cuda")
    gpu, a, w = operands(40, 83, 1300, bits)
    check_product(run(B, (rows, cols, 2), gpu, 40, 83, 1300, bits, dtype, wide[:, :83]), a, w, 1300, dtype)
    assert (wide[:, 83:] == 7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,cols", ROWS + TILES, ids=lambda v: str(v))
def test_nan_stays_in_its_row_and_column_on_every_kernel(B, rows, cols, bits, dtype):
    M, N = (9 if rows == 16 else rows + 40), 100
    for K, slices in ((1024, 1), (700, 1)) + (((2100, 2),) if rows > 32 else ()):
        gpu, a, w = operands(M, N, K, bits)
        ref = run(B, (rows, cols, slices), gpu, M, N, K, bits, dtype)
        codes, scales, packed = (t.clone() for t in gpu)
        if bits == 8:
            codes[1, 600] = 0x7F
        else:
            scales[1, 18] = 255
        groups = -(-K // 512)
        packed.view(-1, groups, 4352)[3, 1, 4096 + 4 * (16 * 2 + 5) + 1] = 255       # feature 53, a block of the second 512 values
        out = run(B, (rows, cols, slices), (codes, scales, packed), M, N, K, bits, dtype)
        hit = torch.zeros(M, N, dtype=torch.bool, device="cuda")
        hit[1], hit[:, 53] = True, True
        assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], ref[~hit])


def few_large_ones(M, N, K, seed):
    """Rows of zeros but for six codes of any magnitude, some of them pairs of the largest with opposite signs, and weights of
    6 and 0.5: every product is a multiple of 2^-10 and below 2^12, so any order of adding six of them in fp32 is exact."""
    r = np.random.RandomState(seed)
    codes = np.zeros((M, -(-K // 128) * 128), np.uint8)
    for m in range(M):
        at = r.randint(0, K) // 8 * 8 + r.permutation(8)[:6] if m % 2 else r.permutation(K)[:6]      # six of eight neighbours, or anywhere
        at = np.minimum(at, K - 1)
        small = r.randint(1, 0x7E, 6)
        small[0], small[1] = 0x7E, 0xFE                                # 448 and -448
        if m % 4 == 1:
            small[2:] = 0x41                                           # 2.25
        elif m % 4 == 3:
            small[2:] = r.choice([0x01, 0x3F, 0x40, 0x41, 0x47], 4)      # 2^-9, 1.875, 2, 2.25, 3.75
        codes[m, at] = small | (r.randint(0, 2, 6) << 7) * (np.arange(6) > 1)
    w = r.choice(np.array([1, 7, 9, 15], np.uint8), (N, codes.shape[1]))        # 0.5, 6, -0.5, -6
    w[:, K:] = 0
    w[0] = np.where(w[0] & 8, 15, 7) * (np.arange(len(w[0])) < K)
    return codes, w


@pytest.mark.parametrize("rows,cols", ROWS + TILES, ids=lambda v: str(v))
def test_fp32_results_drop_nothing(B, rows, cols):
    """small products beside large ones that cancel: equal to the sum in 64 bits, to the bit"""
    K = 1300
    M, N = (16 if rows == 16 else 500), 100
    for seed in range(8 if rows == 16 else 2):
        ca, cw = few_large_ones(M, N, K, seed)
        sa, sw = np.full((M, ca.shape[1] // 32), 127, np.uint8), np.full((N, ca.shape[1] // 32), 127, np.uint8)
        gpu = [torch.from_numpy(x).cuda() for x in (ca, sa, R.pack_weights(cw, sw, N, K))]
        want = R.values(ca, sa, 8) @ R.values(cw, sw, 4).T
        assert (want == want.astype(np.float32)).all()
        got = run(B, (rows, cols, 1), gpu, M, N, K, 8, "fp32").double().cpu().numpy()
        assert np.array_equal(got, want), (np.count_nonzero(got != want), np.abs(got - want).max())


@pytest.mark.parametrize("M,N", [(7, 96), (20, 96), (500, 90)])
def test_bf16_results_cut_what_is_stated(B, M, N):
    """among eight neighbours each product loses less than 2^-13 of the largest, towards zero; eights are added in fp32 and the result is rounded once"""
    K = 1300
    for seed in range(4):
        ca, cw = few_large_ones(M, N, K, 10 + seed)
        sa, sw = np.full((M, ca.shape[1] // 32), 127, np.uint8), np.full((N, ca.shape[1] // 32), 127, np.uint8)
        gpu = [torch.from_numpy(x).cuda() for x in (ca, sa, R.pack_weights(cw, sw, N, K))]
        a, w = R.values(ca, sa, 8), R.values(cw, sw, 4)
        lost = np.zeros((M, N))
        for k in range(0, a.shape[1], 8):
            p = np.abs(a[:, None, k:k + 8] * w[None, :, k:k + 8])
            lost += 2.0 ** -13 * p.max(-1) * np.maximum((p > 0).sum(-1) - 1, 0)
        plan = B.sjd_mx_product_plan(M, N, K)
        got, want = run(B, plan, gpu, M, N, K, 8, "bf16").double().cpu().numpy(), a @ w.T
        room = (lost + K * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T)) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
        assert (np.abs(got - want) <= room).all(), np.max(np.abs(got - want) / room)


def test_what_the_hook_refuses(B):
    gpu, a, w = operands(40, 100, 512, 8)
    for plan in ((48, 64, 1), (64, 65, 1), (64, 256, 1), (64, 64, 3), (64, 64, 0), (64, 64, 8), (16, 16, 1), (32, 96, 1), (32, 16, 2), (32, 80, 1), (32, 0, 1), (0, 0, 1)):
        with pytest.raises(B.SjdError) as e:
            run(B, plan, gpu, 40, 100, 512, 8, "fp32")
        assert e.value.code == B.SJD_EINVAL, plan


def test_a_missing_workspace_is_refused(B):
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = torch.zeros(1, 64, device="cuda")
    cache, scales = (torch.zeros(64 * m, dtype=torch.uint8, device="cuda") for m in (64 * 64, 2))
    M, N, K = 128, 4096, 11008
    assert B.sjd_mx_product_workspace(M, N, K) > 0
    gpu = [torch.zeros(m, dtype=torch.uint8, device="cuda") for m in (M * K, M * K // 32, B.sjd_mx_weights_bytes(N, K))]
    for f in (lambda: B.sjd_kv8_attention(x, cache, scales, n, 1, 1, 1, 64, 2048, 0, 0, torch.zeros_like(x), None),
              lambda: B.sjd_mx_product(8, *gpu, K, torch.zeros(M, N, device="cuda"), None)):
        with pytest.raises(B.SjdError) as e:
            f()
        assert e.value.code == B.SJD_EINVAL
