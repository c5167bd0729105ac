"""What the microscaled operators refuse, before anything reaches a GPU, and the sizes they state (no GPU needed)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import mx_reference as R  # noqa: E402
from paper_2410_01699_amd import binding as B  # noqa: E402

OK, BAD = B.SJD_OK, B.SJD_EINVAL
P = 1 << 20                 # an address that no refused call touches
ODD = P + 8


def call(name, args, **change):
    """the C entry with the named arguments, some changed"""
    a = dict(args, **change)
    return getattr(B._lib, name)(*a.values())


QUANT = dict(format=8, dtype=0, x=P, up=None, ld=64, rows=4, K=64, codes=P, scales=P, stream=None)
NORM = dict(format=8, dtype=0, x=P, ldx=64, resid=P, ldr=64, gain=P, eps=1e-5, rows=4, d=64, codes=P, scales=P, stream=None)
WEIGHTS = dict(dtype=0, W=P, ld=64, N=16, K=64, packed=P, stream=None)
PRODUCT = dict(format=8, codes=P, scales=P, packed=P, M=4, N=16, K=64, dtype=0, C=P, ldc=16, ws=P, ws_bytes=1 << 30, stream=None)
APPEND = dict(dtype=0, k=P, v=P, ld=128, len=P, n_seqs=2, L=4, n_kv=2, hd=64, cap=64, cache=P, scales=P, stream=None)
ATTEND = dict(dtype=0, q=P, ldq=256, cache=P, scales=P, len=P, n_seqs=2, L=4, heads=4, n_kv=2, hd=64, cap=64, window=0, sinks=0, out=P, ldo=256,
              ws=P, ws_bytes=1 << 30, stream=None)

REFUSED = [
    ("sjd_mx_quantize", QUANT, [dict(format=6), dict(dtype=2), dict(dtype=-1), dict(x=None), dict(codes=None), dict(scales=None), dict(ld=63), dict(rows=0),
                                dict(K=0), dict(K=B.SJD_MX_MAX_K + 1, ld=1 << 40), dict(codes=ODD), dict(scales=ODD),
                                dict(rows=2 ** 31 - 1)]),
    ("sjd_mx_rmsnorm", NORM, [dict(format=0), dict(dtype=2), dict(x=None, resid=None), dict(gain=None), dict(codes=None), dict(scales=None), dict(ldx=63),
                              dict(ldr=63), dict(rows=0), dict(rows=-1), dict(d=0), dict(eps=-1.0), dict(eps=float("nan")), dict(codes=ODD), dict(scales=ODD), dict(rows=2 ** 31 - 1)]),
    ("sjd_mx_weights", WEIGHTS, [dict(dtype=2), dict(W=None), dict(packed=None), dict(packed=ODD), dict(ld=63), dict(N=0), dict(K=0), dict(N=2 ** 31 - 1)]),
    ("sjd_mx_product", PRODUCT, [dict(format=5), dict(dtype=2), dict(codes=None), dict(scales=None), dict(packed=None), dict(C=None), dict(M=0), dict(N=0),
                                 dict(K=0), dict(ldc=15), dict(N=2 ** 31 - 1, ldc=2 ** 31), dict(codes=ODD), dict(scales=ODD), dict(packed=ODD)]),
    ("sjd_kv8_append", APPEND, [dict(dtype=2), dict(k=None), dict(v=None), dict(len=None), dict(cache=None), dict(scales=None), dict(cache=ODD), dict(scales=ODD),
                                dict(ld=127), dict(n_seqs=0), dict(n_seqs=1 << 20), dict(L=0), dict(L=65), dict(n_kv=0), dict(n_kv=1 << 20, ld=1 << 40), dict(hd=48),
                                dict(hd=0), dict(hd=512, ld=2048), dict(cap=0), dict(cap=2 ** 31 - 1)]),
    ("sjd_kv8_attention", ATTEND, [dict(dtype=2), dict(q=None), dict(cache=None), dict(scales=None), dict(len=None), dict(out=None), dict(cache=ODD),
                                   dict(scales=ODD), dict(ldq=255), dict(ldo=255), dict(n_seqs=0), dict(L=0), dict(L=65), dict(heads=3), dict(heads=1),
                                   dict(heads=0), dict(hd=80), dict(cap=0), dict(window=-1), dict(sinks=-1), dict(ws=None, cap=2048), dict(ws=ODD, cap=2048), dict(ws_bytes=16, cap=2048)]),
]


@pytest.mark.parametrize("name,args,change", [(n, a, c) for n, a, cs in REFUSED for c in cs], ids=lambda v: v if isinstance(v, str) else "-".join(v) if len(v) < 4 else "")
def test_the_entry_refuses(name, args, change):
    assert call(name, args, **change) == BAD


def test_sizes():
    assert B.sjd_mx_weights_bytes(1, 1) == 4352 and B.sjd_mx_weights_bytes(17, 513) == 4 * 4352
    assert B.sjd_mx_weights_bytes(22016, 4096) == 1376 * 8 * 4352
    n = C.c_size_t()
    for f, bad in (("sjd_mx_weights_bytes", (0, 1)), ("sjd_mx_weights_bytes", (1, 0)), ("sjd_mx_product_workspace", (0, 1, 1)),
                   ("sjd_kv8_attention_workspace", (1, 1, 3, 2, 64, 64)), ("sjd_kv8_attention_workspace", (1, 1, 2, 2, 48, 64))):
        assert getattr(B._lib, f)(*bad, C.byref(n)) == BAD
    assert B._lib.sjd_mx_weights_bytes(1, 1, None) == BAD and B._lib.sjd_mx_product_workspace(1, 1, 1, None) == BAD
    assert B._lib.sjd_kv8_attention_workspace(1, 1, 1, 1, 64, 64, None) == BAD
    # a workspace does not grow with the cache, and short ones need none
    assert B.sjd_kv8_attention_workspace(1, 1, 8, 8, 128, 1 << 20) == B.sjd_kv8_attention_workspace(1, 1, 8, 8, 128, 1025) > 0
    assert B.sjd_kv8_attention_workspace(1, 1, 8, 8, 128, 1024) == 0


def u8(n):
    return torch.empty(n, dtype=torch.uint8)


def test_the_binding_refuses_what_is_not_on_the_gpu():
    x = torch.empty(2, 64)
    for f in (lambda: B.sjd_mx_quantize(8, x, u8(256), u8(8)),
              lambda: B.sjd_mx_rmsnorm(8, x, None, torch.empty(64), 1e-5, u8(256), u8(8)),
              lambda: B.sjd_mx_rmsnorm(8, None, None, torch.empty(64), 1e-5, u8(256), u8(8)),
              lambda: B.sjd_mx_weights(x, u8(4352)),
              lambda: B.sjd_mx_product(8, u8(256), u8(8), u8(4352), 64, torch.empty(2, 16), None),
              lambda: B.sjd_kv8_append(x, x, torch.zeros(2, dtype=torch.int32), 1, 1, 64, 32, u8(8192), u8(4)),
              lambda: B.sjd_kv8_attention(x, u8(8192), u8(4), torch.zeros(2, dtype=torch.int32), 1, 1, 1, 64, 32, 0, 0, x, None)):
        with pytest.raises(B.SjdError) as e:
            f()
        assert e.value.code == BAD


def test_formats_of_the_reference():
    """the tables, rounding and scales that the GPU tests compare with, against torch's own E4M3 and by hand"""
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert ((t == R.table(8)) | (t != t)).all() and R.table(4)[:8].tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    x = torch.cat((torch.linspace(-448, 448, 20011), torch.linspace(-0.1, 0.1, 20011), torch.tensor([17.0, 19.0, 0.0009765625])))
    assert (R.nearest(x.double().numpy(), 8) == x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()).all()
    assert [int(R.nearest(torch.tensor([v]).double().numpy(), 4)[0]) for v in (0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, -5.1)] == [0, 1, 2, 2, 4, 4, 6, 6, 7, 15]
    for a, b8 in ((448.0, 127), (448.5, 128), (224.0, 126), (1.0, 119), (0.0, 0), (2.0 ** -149, 0)):
        assert R.scale_byte(a, 8) == b8 == int(R.scale_bytes(torch.tensor([a]).double().numpy(), 8)[0])


def test_packed_orders_hold_every_value_once():
    k, v = R.cache_at(96)
    assert sorted(k.reshape(-1).tolist() + v.reshape(-1).tolist()) == list(range(64 * 96))
    import numpy as np
    codes = np.random.RandomState(0).randint(0, 16, (21, 640)).astype(np.uint8)
    scales = np.random.RandomState(1).randint(1, 255, (21, 20)).astype(np.uint8)
    w = R.pack_weights(codes, scales, 21, 640).reshape(2, 2, 4352)
    n, kk = 19, 513 + 128 + 64 + 3 - 130                     # feature 19, value 578: group 1, step 0, quarter 2, value 2 of it
    assert kk == 578 and w[1, 1, 16 * (16 * 2 + 3) + 1] & 15 == codes[n, kk] and w[1, 1, 4096 + 4 * (16 * 2 + 3)] == scales[n, 18]


PLANS = {(16, 16 * t, 1) for t in (1, 2, 3, 4, 6)} | {(32, 16 * t, 1) for t in (1, 2, 3, 4)} | {
    (*t, s) for t in ((64, 64), (64, 128), (64, 192), (128, 128), (128, 192), (128, 256), (256, 256)) for s in (1, 2, 3, 4)}


def test_plans_are_kernels_that_exist():
    """every plan is one that the parity entry takes, and its workspace is what the plan's slices need"""
    seen = set()
    for M in (1, 2, 15, 16, 17, 32, 33, 64, 100, 129, 200, 256, 500, 512, 1000, 1024, 2048, 5000, 100000):
        for N in (1, 16, 50, 256, 1536, 4096, 4608, 8192, 12288, 16384, 22016):
            for K in (1, 128, 700, 1536, 4096, 11008, 1 << 17):
                rows, cols, slices = p = B.sjd_mx_product_plan(M, N, K)
                assert p in PLANS and (rows == 16) == (M <= 16) and (rows <= 32 or M > 32), (M, N, K, p)
                assert B.sjd_mx_product_workspace(M, N, K) == (slices * M * (-(-N // 4) * 4) * 4 if slices > 1 else 0)
                seen.add((rows, cols))
    assert len(seen) == 16                                    # no kernel that nothing reaches
    n = C.c_int32()
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, B.SJD_MX_MAX_K + 1)):
        assert B._lib.sjd_mx_product_plan(*bad, C.byref(n), C.byref(n), C.byref(n)) == BAD
    assert B._lib.sjd_mx_product_plan(1, 1, 1, None, C.byref(n), C.byref(n)) == BAD


@pytest.mark.parametrize("size,plan", [((16, 22016, 4096), (16, 96, 1)), ((100, 4096, 4096), (32, 64, 1)), ((100, 8192, 1536), (64, 64, 1)), ((100, 4096, 11008), (64, 128, 4)),
                                       ((200, 4096, 4096), (64, 64, 1)), ((256, 12288, 4096), (64, 192, 1)), ((512, 4096, 4096), (64, 128, 1)),
                                       ((1024, 8192, 1536), (128, 256, 1)), ((2048, 12288, 4096), (128, 192, 1)), ((2048, 22016, 4096), (128, 192, 1))])
def test_plans_of_the_sizes_whose_times_the_source_gives(size, plan):
    """the table beside the plan names the kernel that runs"""
    assert B.sjd_mx_product_plan(*size) == plan


HOOK = dict(rows=64, cols=64, slices=1, format=8, codes=P, scales=P, packed=P, M=40, N=16, K=640, dtype=0, C=P, ldc=16, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [dict(format=5), dict(dtype=2), dict(codes=None), dict(C=None), dict(K=0), dict(ldc=15), dict(codes=ODD), dict(rows=48), dict(cols=80),
                                    dict(cols=256), dict(slices=3), dict(slices=0), dict(rows=16, cols=16), dict(rows=32, cols=96), dict(rows=32, cols=80, M=20),
                                    dict(rows=32, cols=16, slices=2), dict(rows=32, cols=0), dict(M=32), dict(rows=16, cols=96, M=17), dict(rows=0, cols=0),
                                    dict(slices=2, ws=None), dict(slices=2, ws_bytes=16), dict(slices=2, ws=ODD)])
def test_the_parity_entry_refuses(change):
    assert call("sjd_mx_product_test", HOOK, **change) == BAD


def test_what_later_positions_do_to_a_block():
    """the bounds that the header states for earlier codes of a block: kept within 2^13 of the largest magnitude appended to it, rejected ones
    too, else off by at most 2^-16 of that (the reference moves codes as the kernel does, byte for byte)"""
    import numpy as np
    r = np.random.RandomState(4)
    lost = 0
    for case in range(60):
        c = R.Cache(1, 1, 32, 32)
        new = lambda L, e: (r.randn(1, L, 1, 32) * 2.0 ** r.uniform(*e, (1, L, 1, 1))).astype(np.float32).astype(np.float64)
        first = new(4, (-20, 0))
        c.append(first, first, [0], 4)
        before, largest = c.values(0, 0, 4)[0], np.abs(first).max()
        for n, e in ((4, (-3, 12)), (4, (5, 20)), (4, (-9, -2)), (9, (-20, 25))):             # a window, rejected twice, then kept
            x = new(5, e)
            c.append(x, x, [n], 5)
            largest = max(largest, np.abs(x).max())
            off = np.abs(c.values(0, 0, 4)[0] - before)
            assert (off <= 2.0 ** -16 * largest).all() and (off[np.abs(before) >= 2.0 ** -13 * largest] == 0).all()
        lost += np.count_nonzero(off)
    assert lost


@pytest.mark.parametrize("name,args,change", [
    ("sjd_kv8_append", APPEND, dict(L=1 << 28, cap=1 << 28, hd=256, ld=512)),                     # 2^23 + 1 workgroups of 512
    ("sjd_kv8_append", APPEND, dict(L=2 ** 31 - 65, cap=2 ** 31 - 65, hd=64)),
    ("sjd_mx_product", PRODUCT, dict(M=2 ** 31 - 1, N=1 << 17, ldc=1 << 17)),                      # no kernel has a grid for that
    ("sjd_mx_product", PRODUCT, dict(M=2 ** 31 - 1, N=2 ** 31 - 1, ldc=1 << 31)),
    ("sjd_mx_product_test", HOOK, dict(slices=2, M=1 << 20, N=1 << 14, ldc=1 << 14, ws_bytes=1 << 60)),          # 2^32 threads that join
])
def test_launches_that_no_grid_holds_are_refused(name, args, change):
    assert call(name, args, **change) == BAD


def test_workspaces_of_the_widest_products():
    """sizes whose tiles or padded columns pass 32 bits: no size that has wrapped around, an error where no kernel has a grid"""
    for M, N in ((1, 2 ** 31 - 1), (33, 2 ** 31 - 1), (100, 2 ** 31 - 2), (2 ** 31 - 1, 1)):
        assert B.sjd_mx_product_workspace(M, N, 4096) <= 4 * M * 2 ** 31 * 4
        assert B.sjd_mx_product_plan(M, N, 4096) in PLANS
    for f in (B.sjd_mx_product_workspace, B.sjd_mx_product_plan):
        with pytest.raises(B.SjdError) as e:
            f(2 ** 31 - 1, 2 ** 31 - 1, 4096)
        assert e.value.code == BAD


def test_a_workspace_that_is_needed_and_missing_is_an_error_of_the_library():
    with pytest.raises(B.SjdError) as e:
        B._workspace(0, None, 64)
    assert e.value.code == BAD
    assert B._workspace(0, None, 0) == (None, 0)


def test_a_stream_of_another_device_is_refused():
    class Stream:
        cuda_stream, device_index = 5, 1

    assert B._on(1, Stream) == 5 and B._on(1, None) is None
    with pytest.raises(B.SjdError) as e:
        B._on(0, Stream)
    assert e.value.code == BAD
