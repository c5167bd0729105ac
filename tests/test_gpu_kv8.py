"""The 8-bit cache and the attention over it (GPU only), against mx_reference.

Appending is exact, so the bytes are equal.  Attention in fp32: a score is a sum of hd products of fp32 queries held to 2^-22 and exact
keys, off by at most d = (2^-22 + (hd + 8) 2^-24) sum |q k| / sqrt(hd); probabilities are off by a factor of e^(2 d) and 2^-20
(fp16 pairs, exponentials, rescaling), the output by that of the largest |v| it averages.  bf16 results: probabilities in one fp16 (2^-11), and
2^-8 of the output for its own rounding.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import mx_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_01699_amd import binding
    return binding


def rnd(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def lengths(n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


class Pair:
    """a cache on the GPU and its reference"""

    def __init__(self, B, n_seqs, n_kv, hd, cap, dtype="fp32"):
        self.B, self.shape, self.dtype = B, (n_seqs, n_kv, hd, cap), dtype
        self.ref = R.Cache(n_seqs, n_kv, hd, cap)
        self.codes, self.scales = torch.from_numpy(self.ref.codes.copy()).cuda(), torch.from_numpy(self.ref.scales.copy()).cuda()

    def append(self, n, L, seed=0, change=None):
        n_seqs, n_kv, hd, cap = self.shape
        kv = rnd(seed, n_seqs, L, 2, n_kv, hd)
        kv = kv * 2.0 ** torch.randint(-4, 5, (n_seqs, L, 1, 1, 1), generator=torch.Generator().manual_seed(seed + 1))
        if change:
            change(kv)
        kv = kv.to(TYPES[self.dtype])
        rows = kv.reshape(n_seqs * L, -1).cuda()
        self.B.sjd_kv8_append(rows[:, :n_kv * hd], rows[:, n_kv * hd:], lengths(n), L, n_kv, hd, cap, self.codes, self.scales)
        k = kv.double().numpy()
        self.ref.append(k[:, :, 0], k[:, :, 1], n, L)

    def same(self):
        assert np.array_equal(self.scales.cpu().numpy(), self.ref.scales)
        assert np.array_equal(self.codes.cpu().numpy(), self.ref.codes)

    def attend(self, n, L, n_heads, window=0, sinks=0, dtype="fp32", seed=5, change=None, pad=0, stream=None):
        n_seqs, n_kv, hd, cap = self.shape
        q = rnd(seed, n_seqs * L, n_heads * hd + pad)
        if change:
            change(q)
        q = q.to(TYPES[dtype])
        out = torch.full((n_seqs * L, n_heads * hd + pad), 7.0, dtype=TYPES[dtype], device="cuda")
        ws = torch.full((self.B.sjd_kv8_attention_workspace(n_seqs, L, n_heads, n_kv, hd, cap),), 0xFF, dtype=torch.uint8, device="cuda")
        cols = n_heads * hd
        self.B.sjd_kv8_attention(q.cuda()[:, :cols], self.codes, self.scales, lengths(n), L, n_heads, n_kv, hd, cap, window, sinks, out[:, :cols], ws)
        assert (out[:, cols:] == 7).all()
        q = q[:, :cols].double().numpy().reshape(n_seqs, L, n_heads, hd)
        with np.errstate(invalid="ignore"):
            want, mag, top = R.attention(self.ref, q, n, L, n_heads, window, sinks)
        got = out[:, :cols].double().cpu().numpy().reshape(n_seqs, L, n_heads, hd)
        return got, want, mag, top

    def check(self, n, L, n_heads, window=0, sinks=0, dtype="fp32", **kw):
        got, want, mag, top = self.attend(n, L, n_heads, window, sinks, dtype, **kw)
        hd, cap = self.shape[2:]
        d = (2.0 ** -22 + (hd + 8) * 2.0 ** -24) * mag
        room = (np.expm1(2 * d) + 2.0 ** -20 + (2.0 ** -11 if dtype == "bf16" else 0)) * top
        room = room + (2.0 ** -8 * (np.abs(want) + room) if dtype == "bf16" else 0)
        for b, m in enumerate(n):
            if m < 0 or m + L > cap:
                assert (got[b] == 7).all()
            else:
                assert np.isfinite(got[b]).all()
                assert (np.abs(got[b] - want[b]) <= room[b]).all(), (b, np.max(np.abs(got[b] - want[b]) / room[b]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("n,L", [([0, 0], 1), ([0, 5], 31), ([31, 32], 1), ([33, 63], 2), ([1, 40], 70)])
def test_append_to_the_byte(B, n, L, hd, dtype):
    c = Pair(B, 2, 3, hd, 128, dtype)
    if max(n):
        c.append([0, 0], max(n), seed=20)
    c.append(n, L, seed=21)
    c.same()


def test_windows_are_appended_over_rejected_ones(B):
    """as in decoding: a window of 16, of which some are kept, then the next one over the rest"""
    c, n = Pair(B, 2, 2, 64, 160), [3, 30]
    c.append([0, 0], 30)
    for i, kept in enumerate([(1, 16), (7, 2), (16, 1), (5, 5), (0, 11)]):
        c.append(n, 16, seed=30 + i)
        c.same()
        n = [a + k for a, k in zip(n, kept)]
    c.append(n, 1, seed=40)
    c.append(n, 1, seed=40)                      # the same again
    c.same()


def test_scales_grow_shrink_and_vanish(B):
    def to(f):
        def change(kv):
            kv.mul_(f)
        return change

    c = Pair(B, 1, 1, 64, 64)
    for i, (n, f) in enumerate([(0, 1.0), (4, 2.0 ** 40), (8, 2.0 ** -100), (4, 2.0 ** -20), (0, 0.0), (2, 2.0 ** -130), (6, 2.0 ** 120), (33, 1.0)]):
        c.append([n], 4, seed=50 + i, change=to(f))
        c.same()


def test_a_sequence_without_room_sits_out(B):
    c = Pair(B, 5, 2, 64, 100)
    c.append([0, 97, -1, 96, 2 ** 31 - 1], 4)
    c.same()
    c = Pair(B, 4, 1, 64, 70)
    c.append([0] * 4, 66)
    c.check([66, -1, 67, 2], 4, 1)


def test_infinities_and_nan_stay_in_their_places(B):
    def change(kv):
        kv[0, 3, 0, 0, 5], kv[0, 4, 0, 0, 6], kv[0, 5, 1, 1, 7] = float("inf"), float("nan"), -float("inf")

    c = Pair(B, 1, 2, 64, 64)
    c.append([0], 20, change=change)
    c.same()
    c.append([20], 9, seed=9)
    c.same()


@pytest.mark.parametrize("off", [1, 4])
def test_append_from_rows_of_a_wider_matrix(B, off):
    n_kv, hd, L = 2, 64, 7
    rows = rnd(3, 2 * L, off + 2 * n_kv * hd + 3).cuda()
    k, v = rows[:, off:off + n_kv * hd], rows[:, off + n_kv * hd:off + 2 * n_kv * hd]
    ref = R.Cache(2, n_kv, hd, 64)
    codes, scales = torch.from_numpy(ref.codes.copy()).cuda(), torch.from_numpy(ref.scales.copy()).cuda()
    B.sjd_kv8_append(k, v, lengths([0, 0]), L, n_kv, hd, 64, codes, scales)
    ref.append(*(x.double().cpu().numpy().reshape(2, L, n_kv, hd) for x in (k, v)), [0, 0], L)
    assert np.array_equal(codes.cpu().numpy(), ref.codes) and np.array_equal(scales.cpu().numpy(), ref.scales)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("n,L,heads,n_kv", [([0, 0], 1, 2, 2), ([0, 7], 5, 4, 2), ([100, 31], 16, 2, 2), ([200, 150], 9, 8, 2), ([64, 90], 40, 3, 1)])
def test_attention(B, n, L, heads, n_kv, hd, dtype):
    c = Pair(B, 2, n_kv, hd, 288)
    c.append([0, 0], max(n) + L, seed=60)
    c.check(n, L, heads, dtype=dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (32, 0), (33, 32), (40, 33), (64, 100), (1000, 5), (100, 1000), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("n,L,heads", [([0, 3, 250], 1, 1), ([300, 95, 64], 20, 2)])
def test_sliding_window_and_sinks(B, n, L, heads, window, sinks, dtype):
    c = Pair(B, 3, 1, 64, 320)
    c.append([0] * 3, 320, seed=61)
    c.check(n, L, heads, window, sinks, dtype)


@pytest.mark.parametrize("n,L,heads,n_kv,window,sinks", [([3000, 0, 777], 1, 4, 4, 0, 0), ([2048, 2047], 3, 16, 2, 0, 0), ([4001], 37, 2, 1, 0, 0), ([4000, 100], 6, 4, 1, 1500, 70)])
def test_long_caches_are_split_and_joined(B, n, L, heads, n_kv, window, sinks):
    c = Pair(B, len(n), n_kv, 64, 4064)
    c.append([0] * len(n), 4064, seed=62)
    c.check(n, L, heads, window, sinks)
    c.check(n, L, heads, window, sinks, "bf16")


def test_many_sequences(B):
    """more (sequence, rows) pairs than lanes of a wave; lengths from none to long"""
    n = [(37 * i) % 200 if i % 9 else -1 for i in range(150)]
    c = Pair(B, 150, 1, 32, 224)
    c.append([0] * 150, 200, seed=63)
    c.append(n, 3, seed=64)
    c.same()
    c.check(n, 3, 2)


def test_pairs_that_fill_the_chip_are_not_split(B):
    assert B.sjd_kv8_attention_workspace(16, 1, 32, 32, 64, 96) == 0
    c = Pair(B, 16, 32, 64, 96)
    c.append([0] * 16, 66, seed=65)
    c.check([65 - 3 * i for i in range(16)], 1, 32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_one_long_sequence_among_short_ones(B, dtype):
    """pairs enough to fill the chip, of which one holds most of the positions: its walk is cut"""
    n_seqs, n_kv, hd, cap = 5, 48, 32, 8224
    assert B.sjd_kv8_attention_workspace(n_seqs, 2, n_kv, n_kv, hd, cap) > 0 == B.sjd_kv8_attention_workspace(n_seqs, 40, n_kv, n_kv, hd, cap)
    c = Pair(B, n_seqs, n_kv, hd, cap)
    c.append([-1, -1, 0, -1, -1], 3000, seed=73)                  # (append in pieces: the reference's arrays)
    c.append([-1, -1, 3000, -1, -1], 3000, seed=74)
    c.append([0, 0, -1, 0, 0], 300, seed=75)
    for n in ([40, 299, 5998, 0, -1], [7, 200, 100, 0, 298]):     # (the second: nothing to cut)
        c.check(n, 2, n_kv, dtype=dtype)
    c.check([40, 299, 5998, 0, 250], 2, n_kv, window=2500, sinks=40, dtype=dtype)


def test_scales_of_blocks_far_apart(B):
    """keys and values of whole blocks far smaller and larger than their neighbours', and blocks of zeros"""
    def change(kv):
        for blk, e in enumerate([0, 40, -60, 0, 60, -30]):
            kv[:, 32 * blk:32 * blk + 32, 1] *= 2.0 ** e
        for blk, e in enumerate([0, -20, 2, -90, 1, 0]):
            kv[:, 32 * blk:32 * blk + 32, 0] *= 2.0 ** e
        kv[:, 96:128] = 0

    for hd in (64, 128):
        c = Pair(B, 1, 2, hd, 192)
        c.append([0], 192, seed=66, change=change)
        for n in (10, 50, 90, 120, 180):
            c.check([n], 3, 2)
        # the large ones hidden by the window, so that the small ones are all there is
        c.check([90], 2, 2, window=20)
        c.check([190], 2, 2, window=20)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd,heads", [(64, 1), (128, 3)])
@pytest.mark.parametrize("kind", ["rising", "falling", "large and unlikely", "any"])
def test_value_scales_that_leave_their_neighbourhood(B, kind, hd, heads, dtype):
    """Several blocks to a wave, whose value scales wander off from the first one's.  The error is held to the mean of |v| under the
    probabilities: those are off as above, and a sum of n products in fp32 by n 2^-24 of it."""
    n, L, blocks = 1000, 3, 32
    r = np.random.RandomState(7)
    ev = {"rising": 1.5 * np.arange(blocks), "falling": -1.5 * np.arange(blocks), "large and unlikely": 24 * (np.arange(blocks) >= 12), "any": r.randint(-40, 40, blocks)}[kind]
    ev = np.floor(ev)

    def change(kv):
        for blk in range(blocks):
            kv[:, 32 * blk:32 * blk + 32, 1] *= 2.0 ** ev[blk]
        kv[:, :, 0, :, 0] = 0.0
        if kind == "large and unlikely":                        # scores lower by 20 log 2 or so (queries have 8 there)
            kv[:, 32 * 12:, 0, :, 0] = -20 * np.log(2) * hd ** 0.5 / 8

    def eight(q):
        q[:, ::hd] = 8.0

    c = Pair(B, 1, 1, hd, 1024)
    c.append([0], n + L, seed=76, change=change)
    got, want, mag, _ = c.attend([n], L, heads, dtype=dtype, change=eight)

    class Magnitudes:
        codes, hd, cap = c.ref.codes, c.ref.hd, c.ref.cap

        def values(self, *a):
            k, v = c.ref.values(*a)
            return k, np.abs(v)

    q = rnd(5, L, heads * hd)
    eight(q)
    mean, _, _ = R.attention(Magnitudes(), q.to(TYPES[dtype]).double().numpy().reshape(1, L, heads, hd), [n], L, heads, 0, 0)
    d = (2.0 ** -22 + (hd + 8) * 2.0 ** -24) * mag
    room = (np.expm1(2 * d) + 2.0 ** -20 + (n + L) * 2.0 ** -24 + (2.0 ** -11 if dtype == "bf16" else 0)) * mean
    room = room + (2.0 ** -8 * (np.abs(want) + room) if dtype == "bf16" else 0)
    assert np.isfinite(got).all() and (np.abs(got - want) <= room).all(), np.max(np.abs(got - want) / room)


def test_queries_of_any_magnitude(B):
    def change(q):
        q[0] *= 2.0 ** -100
        q[1] *= 2.0 ** 3
        q[2] = 0
        q[3, ::2] *= 2.0 ** -20

    c = Pair(B, 1, 1, 64, 64)
    c.append([0], 40, seed=67)
    c.check([36], 4, 1, change=change)


def test_what_is_masked_does_not_reach_the_output(B):
    """positions behind the window, and those that a row's mask hides, hold NaN; the scale of the block does not know them"""
    n, L = 70, 8

    def change(kv):
        kv[0, 5], kv[0, 40], kv[0, 77, :, :, ::3] = float("nan"), float("inf"), float("nan")      # sinks' edge, in front of the window, the last position

    for hd, heads in ((64, 1), (128, 3)):
        c = Pair(B, 1, 1, hd, 96)
        c.append([0], 78, seed=68, change=change)
        blk = c.codes.view(-1, 64 * hd)[2]
        at_k, at_v = (torch.from_numpy(a).cuda() for a in R.cache_at(hd))
        blk[at_k[14:].reshape(-1)] = 0x7F                                     # positions 78 .. 95
        blk[at_v[14:].reshape(-1)] = 0xFF
        got, want, mag, top = c.attend([n], L, heads, window=20, sinks=5)
        seen = [i for i in range(L) if i < 7]                                 # the last query sees position 77
        assert np.isfinite(got[0, seen]).all() and np.abs(got[0, seen] - want[0, seen]).max() < 1e-4
        assert np.isnan(got[0, 7]).all()                                      # a NaN key: every probability
        got, want, mag, top = c.attend([n], L, heads, window=20, sinks=6)     # position 5 comes into sight
        assert np.isnan(got).all()


def test_a_visible_nan_value_is_nan_where_it_is_seen(B):
    def change(kv):
        kv[0, 30, 1, 0, 9] = float("nan")

    c = Pair(B, 1, 1, 64, 64)
    c.append([0], 40, seed=69, change=change)
    got, want, _, _ = c.attend([28], 4, 1)                                    # queries at 28 .. 31
    assert np.isfinite(got[0, :2]).all() and np.isnan(got[0, 2:, 0, 9]).all()
    assert np.isfinite(np.delete(got[0, 2:], 9, axis=-1)).all()
    assert np.abs(got[0, :2] - want[0, :2]).max() < 1e-4
    got, _, _, _ = c.attend([35], 1, 1)                                       # the whole block visible
    assert np.isnan(got[0, 0, 0, 9]) and np.isfinite(np.delete(got[0, 0, 0], 9)).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_nan_in_one_split_of_a_long_walk(B, dtype):
    def change(kv):
        kv[0, 100, 1, 0, 9], kv[0, 200, 0, 1, 3] = float("nan"), float("nan")           # a value of head 0, a key of head 1

    c = Pair(B, 1, 3, 64, 4096)
    c.append([0], 4010, seed=75, change=change)
    got, want, _, _ = c.attend([4000], 2, 3, dtype=dtype)
    assert np.isnan(got[0, :, 0, 9]).all() and np.isfinite(np.delete(got[0, :, 0], 9, axis=-1)).all()
    assert np.isnan(got[0, :, 1]).all() and np.isfinite(got[0, :, 2]).all()
    c.check([4000], 2, 3, window=3000, sinks=32, dtype=dtype)                           # both hidden


def test_a_bad_query_row_stays_alone(B):
    def change(q):
        q[3, 7], q[17, 20] = float("nan"), float("inf")

    c = Pair(B, 1, 1, 64, 96)
    c.append([0], 90, seed=70)
    a, _, _, _ = c.attend([60], 30, 1)
    b, _, _, _ = c.attend([60], 30, 1, change=change)
    keep = np.delete(np.arange(30), [3, 17])
    assert np.array_equal(a[0, keep], b[0, keep]) and np.isnan(b[0, [3, 17]]).all()


@pytest.mark.parametrize("pad", [3, 8])
def test_rows_of_wider_matrices(B, pad):
    c = Pair(B, 2, 2, 64, 64)
    c.append([0, 0], 50, seed=71)
    for dtype in TYPES:
        c.check([30, 44], 5, 4, dtype=dtype, pad=pad)


def test_caches_of_more_than_4_gib(B):
    """the last sequence's last positions, seen through a window, give what a short cache gives that holds the same"""
    n_seqs, n_kv, hd, cap, L, window = 3, 8, 256, 393216, 5, 70
    assert n_seqs * n_kv * (cap // 32) * 64 * hd > 2 ** 32
    big = (torch.zeros(n_seqs, n_kv, cap // 32, 64 * hd, dtype=torch.uint8, device="cuda"), torch.zeros(n_seqs, n_kv, cap // 32, 2, dtype=torch.uint8, device="cuda"))
    c = Pair(B, 1, n_kv, hd, 192)
    kv = rnd(90, 160, 2 * n_kv * hd)
    end = cap - 192
    for rows, small, large in ((kv[:160], [0], end), (rnd(91, L, 2 * n_kv * hd), [160], end + 160)):
        k, v = (rows[:, i * n_kv * hd:(i + 1) * n_kv * hd].cuda() for i in range(2))
        B.sjd_kv8_append(k, v, lengths(small), len(rows), n_kv, hd, 192, c.codes, c.scales)
        every = torch.zeros(n_seqs * len(rows), 2 * n_kv * hd, device="cuda")
        every[-len(rows):] = rows.cuda()
        B.sjd_kv8_append(every[:, :n_kv * hd], every[:, n_kv * hd:], lengths([-1, -1, large]), len(rows), n_kv, hd, cap, *big)
    q = rnd(92, n_seqs * L, n_kv * hd).cuda()
    outs = []
    for cache, n, m, x in (((c.codes, c.scales), [160], 192, q[-L:]), (big, [-1, -1, end + 160], cap, q)):
        out = torch.full_like(x, 7.0)
        ws = torch.empty(B.sjd_kv8_attention_workspace(len(n), L, n_kv, n_kv, hd, m), dtype=torch.uint8, device="cuda")
        B.sjd_kv8_attention(x, *cache, lengths(n), L, n_kv, n_kv, hd, m, window, 0, out, ws)
        outs.append(out)
    assert (outs[1][:-L] == 7).all()
    assert torch.equal(outs[0], outs[1][-L:])             # (the same blocks in the same order)


def test_two_attentions_at_the_same_time(B):
    """two streams with a cache and a workspace each, long enough to be split; an append to the one while the other is read"""
    n_kv, hd, cap, n, L = 4, 64, 4096, 4000, 3
    caches = [Pair(B, 1, n_kv, hd, cap) for _ in range(2)]
    qs, ref, wss = [], [], []
    need = B.sjd_kv8_attention_workspace(1, L, n_kv, n_kv, hd, cap)
    assert need > 0
    new = rnd(95, L, 2 * n_kv * hd).cuda()

    def step(c, q, ws, out, stream):
        B.sjd_kv8_append(new[:, :n_kv * hd], new[:, n_kv * hd:], length, L, n_kv, hd, cap, c.codes, c.scales, stream=stream)
        B.sjd_kv8_attention(q, c.codes, c.scales, length, L, n_kv, n_kv, hd, cap, 0, 0, out, ws, stream=stream)

    length = lengths([n])
    for i, c in enumerate(caches):
        c.append([0], n, seed=93 + i)
        qs.append(rnd(97 + i, L, n_kv * hd).cuda())
        wss.append(torch.empty(need, dtype=torch.uint8, device="cuda"))
        ref.append(torch.empty_like(qs[-1]))
        step(c, qs[-1], wss[-1], ref[-1], None)
    outs, streams = [torch.zeros_like(r) for r in ref], [torch.cuda.Stream() for _ in ref]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, q, ws, out, s in zip(caches, qs, wss, outs, streams):
            step(c, q, ws, out, s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, ref))


def test_a_layer_step_is_captured_and_replayed(B):
    """append, attend and advance in a graph, replayed as the cache grows; every replay equals eager calls, on a side stream too"""
    n_seqs, n_kv, heads, hd, cap, L = 2, 2, 4, 64, 640, 4
    ref = Pair(B, n_seqs, n_kv, hd, cap)
    codes, scales, n = ref.codes, ref.scales, lengths([0, 37])
    rows, q = torch.empty(n_seqs * L, 2 * n_kv * hd, device="cuda"), torch.empty(n_seqs * L, heads * hd, device="cuda")
    kv = rnd(1, n_seqs * 37, 2 * n_kv * hd).cuda()
    B.sjd_kv8_append(kv[:, :n_kv * hd], kv[:, n_kv * hd:], lengths([0, 0]), 37, n_kv, hd, cap, codes, scales)
    out, ws = torch.empty_like(q), torch.empty(B.sjd_kv8_attention_workspace(n_seqs, L, heads, n_kv, hd, cap), dtype=torch.uint8, device="cuda")

    def step(codes, scales, n, out, ws, stream):
        B.sjd_kv8_append(rows[:, :n_kv * hd], rows[:, n_kv * hd:], n, L, n_kv, hd, cap, codes, scales, stream=stream)
        B.sjd_kv8_attention(q, codes, scales, n, L, heads, n_kv, hd, cap, 0, 0, out, ws, stream=stream)

    e = [t.clone() for t in (codes, scales, n, out, ws)]
    rows.zero_(); q.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(codes, scales, n, out, ws, torch.cuda.current_stream())
        n += L
    side = torch.cuda.Stream()
    for i in range(130):
        rows.copy_(rnd(100 + i, *rows.shape)); q.copy_(rnd(300 + i, *q.shape))
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            step(*e, side)
            e[2] += L
        torch.cuda.synchronize()
        assert torch.equal(out, e[3]) and torch.equal(codes, e[0]) and torch.equal(scales, e[1]) and torch.equal(n, e[2])


def test_a_decoder_layer_of_these_operators(B):
    """norm, QKV, append, attention, O, norm, gate/up, SwiGLU, down, for prompts and then windows of two sequences, against the same
    layer in 64 bits on the values that each operator was handed"""
    d, heads, n_kv, hd, F, cap, L, n_seqs = 256, 4, 2, 64, 320, 96, 9, 2
    w = {k: 0.05 * rnd(i, *s) for i, (k, s) in enumerate(dict(qkv=((heads + 2 * n_kv) * hd, d), o=(d, heads * hd), gu=(2 * F, d), down=(d, F)).items())}
    packed, wv = {}, {}
    for k, x in w.items():
        packed[k] = torch.empty(B.sjd_mx_weights_bytes(*x.shape), dtype=torch.uint8, device="cuda")
        B.sjd_mx_weights(x.cuda(), packed[k])
        wv[k] = R.values(*R.quantise(x.double().numpy(), 4), 4)
    cache = Pair(B, n_seqs, n_kv, hd, cap)
    gain = torch.ones(d, device="cuda")

    def linear(name, codes, scales, rows, K):
        out = torch.empty(rows, w[name].shape[0], device="cuda")
        ws = torch.empty(B.sjd_mx_product_workspace(rows, out.shape[1], K), dtype=torch.uint8, device="cuda")
        B.sjd_mx_product(8, codes, scales, packed[name], K, out, ws)
        want = R.values(codes.cpu().numpy(), scales.cpu().numpy(), 8) @ wv[name].T
        got = out.double().cpu().numpy()
        assert np.linalg.norm(got - want) <= 1e-6 * np.linalg.norm(want)
        return out

    def coded(rows, K):
        return torch.empty(rows, up128(K), dtype=torch.uint8, device="cuda"), torch.empty(rows, up128(K) // 32, dtype=torch.uint8, device="cuda")

    for n, L in (([0, 0], 30), ([30, 25], 9), ([33, 34], 9)):
        rows = n_seqs * L
        x, resid = rnd(80 + L, rows, d).cuda(), torch.zeros(rows, d, device="cuda")
        codes, scales = coded(rows, d)
        B.sjd_mx_rmsnorm(8, x, resid, gain, 1e-5, codes, scales)
        qkv = linear("qkv", codes, scales, rows, d)
        q, k, v = qkv[:, :heads * hd], qkv[:, heads * hd:(heads + n_kv) * hd], qkv[:, (heads + n_kv) * hd:]
        B.sjd_kv8_append(k, v, lengths(n), L, n_kv, hd, cap, cache.codes, cache.scales)
        cache.ref.append(*(t.double().cpu().numpy().reshape(n_seqs, L, n_kv, hd) for t in (k, v)), n, L)
        cache.same()
        att = torch.empty(rows, heads * hd, device="cuda")
        ws = torch.empty(B.sjd_kv8_attention_workspace(n_seqs, L, heads, n_kv, hd, cap), dtype=torch.uint8, device="cuda")
        B.sjd_kv8_attention(q, cache.codes, cache.scales, lengths(n), L, heads, n_kv, hd, cap, 0, 0, att, ws)
        want, _, _ = R.attention(cache.ref, q.double().cpu().numpy().reshape(n_seqs, L, heads, hd), n, L, heads, 0, 0)
        assert np.linalg.norm(att.double().cpu().numpy().reshape(want.shape) - want) <= 2e-6 * np.linalg.norm(want)
        codes, scales = coded(rows, heads * hd)
        B.sjd_mx_quantize(8, att, codes, scales)
        o = linear("o", codes, scales, rows, heads * hd)
        codes, scales = coded(rows, d)
        B.sjd_mx_rmsnorm(8, o, resid, gain, 1e-5, codes, scales)
        assert torch.equal(resid, x + o)
        gu = linear("gu", codes, scales, rows, d)
        codes, scales = coded(rows, F)
        B.sjd_mx_quantize(8, gu[:, :F], codes, scales, up=gu[:, F:])
        h = gu.double().cpu().numpy()
        y = h[:, :F] / (1 + np.exp(-h[:, :F])) * h[:, F:]
        got = R.values(codes.cpu().numpy(), scales.cpu().numpy(), 8)[:, :F]
        assert np.linalg.norm(got - y) <= 2.0 ** -4 * np.linalg.norm(y)
        linear("down", codes, scales, rows, F)


def up128(n):
    return -(-n // 128) * 128


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("scales", ["near", "apart"])
@pytest.mark.parametrize("e", [18, 22, 24, 25, 26, 30, 60, 110])
def test_scores_beyond_any_fraction(B, e, scales, dtype):
    """Queries of 2^e and -2^e in one place, keys of four bits there: scores are exact, those that are largest are equal, all others are
    lower by 2^e / (8 sqrt(hd)) and more and have no weight.  What is left is the mean of the values at the largest, off by the sums,
    the common factor and one division: 2^-20 of the largest value.  bf16: the equal weights w = 2^x, where x is 12 only up to the rounding of a
    reference of 2^e, are summed as they are and multiplied as one fp16, so the mean is off by fp16(w) / w, up to 2^-11; and it is rounded once more."""
    hd, n, L = 64, 1500, 4
    r = np.random.RandomState(e)

    def change(kv):
        p = kv.shape[1]
        kv[:, :, 0] = 0
        kv[0, :, 0, :, 0] = torch.from_numpy(1 + np.minimum(r.randint(0, 5, (p, 2)) + np.arange(p)[:, None] // 400, 7) / 8)      # rising
        kv[:, :, 1] = rnd(e, *kv[:, :, 1].shape)
        if scales == "apart":
            for blk in range(p // 32 + 1):
                kv[:, 32 * blk:32 * blk + 32, 1] *= 2.0 ** (9 * (blk % 5))

    def only_one_place(q):
        s = torch.tensor([1.0, -1.0, -1.0, 1.0])[:, None]
        q.zero_()
        q[:, ::hd] = s * 2.0 ** e

    for cap, m, window in ((1600, n, 0), (1600, n, 700), (256, 150, 0), (4096, n, 0)):
        c = Pair(B, 1, 2, hd, cap)
        c.append([0], m + L, seed=80, change=change)
        got, want, _, top = c.attend([m], L, 4, window=window, dtype=dtype, change=only_one_place)
        room = (2.0 ** -20 + (2.0 ** -11 if dtype == "bf16" else 0)) * top
        room = room + (2.0 ** -8 * (np.abs(want) + room) if dtype == "bf16" else 0)
        assert np.isfinite(got).all(), (cap, m, window)
        assert (np.abs(got - want) <= room).all(), (cap, m, window, np.max(np.abs(got - want) / room))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [64, 256])
@pytest.mark.parametrize("e", [-100, -110, -116, -122, -128, -134])
def test_values_near_the_smallest(B, e, hd, dtype):
    """outputs down to the types' subnormals, whole walks and joined ones; below 2^-126 an fp32 result is rounded to 2^-150, a bf16 one to 2^-134"""
    def change(kv):
        kv[:, :, 1] = rnd(81, *kv[:, :, 1].shape) * 2.0 ** e

    for cap, n, L, window in ((256, 100, 3, 0), (2048, 1400, 2, 0), (2048, 1300, 2, 500)):
        c = Pair(B, 1, 1, hd, cap)
        c.append([0], n + L, seed=81, change=change)
        got, want, mag, top = c.attend([n], L, 2, window=window, dtype=dtype)
        d = (2.0 ** -22 + (hd + 8) * 2.0 ** -24) * mag
        room = (np.expm1(2 * d) + 2.0 ** -20 + (2.0 ** -11 if dtype == "bf16" else 0)) * top + 2.0 ** -149
        room = room + (2.0 ** -8 * (np.abs(want) + room) + 2.0 ** -134 if dtype == "bf16" else 0)
        assert (np.abs(got - want) <= room).all(), (cap, np.max(np.abs(got - want) / room))
        assert np.abs(want).max() > 2.0 ** (e - 6)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sign", [1, -1])
def test_the_largest_finite_values_stay_when_their_block_grows(B, sign, dtype):
    """Values from 248 * 2^120 on are kept as 256 * 2^120 = 2^128, which no float32 holds: the next window in their block keeps the code.
    And with such a value among rejected ones only."""
    big = sign * float(torch.finfo(TYPES[dtype]).max)
    for at, n, what in ((2, 8, 1.0), (2, 8, -big), (9, 8, 1.0), (2, 8, float("inf")), (3, 31, 2.0 ** -60)):
        def first(kv):
            kv[0, at], kv[0, at + 1] = big, 250 * 2.0 ** 120 * sign

        def second(kv):
            kv[0, 1] = what

        c = Pair(B, 1, 2, 64, 64, dtype)
        c.append([0], max(n, 12), seed=82, change=first)
        c.same()
        with np.errstate(over="ignore"):
            c.append([n], 5, seed=83, change=second)
            c.same()
            c.append([n + 2], 5, seed=84)
        c.same()


def test_a_walk_is_cut_and_whole_from_replay_to_replay(B):
    """one graph over a long cache: lengths from one to many splits, and sequences that sit out, between its replays"""
    n_seqs, n_kv, heads, hd, cap, L = 2, 2, 4, 64, 4096, 3
    c = Pair(B, n_seqs, n_kv, hd, cap)
    c.append([0, 0], cap)
    n = lengths([0, 0])
    q = rnd(90, n_seqs * L, heads * hd).cuda()
    out, eager = torch.empty_like(q), torch.empty_like(q)
    ws = [torch.empty(B.sjd_kv8_attention_workspace(n_seqs, L, heads, n_kv, hd, cap), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def attend(out, ws, stream=None):
        B.sjd_kv8_attention(q, c.codes, c.scales, n, L, heads, n_kv, hd, cap, 0, 0, out, ws, stream=stream)

    mark = 7.1                                  # (no value of the cache: a query that sees one position gives its codes' values)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        attend(out, ws[0], torch.cuda.current_stream())
    for m in ([0, 0], [4000, 10], [10, 1500], [-1, 3000], [4093, 4093], [4094, 700], [-1, -1], [1000, 1000]):
        n.copy_(lengths(m))
        out.fill_(mark); eager.fill_(mark); ws[0].fill_(0xFF); ws[1].fill_(0xFF)
        attend(eager, ws[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), m
        for b, k in enumerate(m):
            rows = out[b * L:(b + 1) * L]
            left = rows == mark
            assert left.all() if k < 0 or k + L > cap else torch.isfinite(rows).all() and not left.any(), m


@pytest.mark.parametrize("n_kv", [1, 4])
@pytest.mark.parametrize("byte", [5, 27, 127, 240])
def test_sums_of_millions_keep_their_bits(B, byte, n_kv):
    """All weights are 2^12 and all values 1.5: sums of up to 2^24 / 1.5 of them are exact in fp32, partial ones added in trees keep 2^-23
    each, and the mean is the value, also where 2^d over the sum of weights would be subnormal"""
    hd, n = 32, 3000001
    cap, at_v = n + 2, R.cache_at(hd)[1]
    codes = torch.zeros(1, n_kv, -(-cap // 32), 64 * hd, dtype=torch.uint8, device="cuda")
    codes[..., torch.from_numpy(at_v.reshape(-1)).cuda()] = 0x3C
    scales = torch.full((1, n_kv, codes.shape[2], 2), byte, dtype=torch.uint8, device="cuda")
    q, out = torch.ones(1, n_kv * hd, device="cuda"), torch.empty(1, n_kv * hd, device="cuda")
    ws = torch.empty(B.sjd_kv8_attention_workspace(1, 1, n_kv, n_kv, hd, cap), dtype=torch.uint8, device="cuda")
    B.sjd_kv8_attention(q, codes, scales, lengths([n]), 1, n_kv, n_kv, hd, cap, 0, 0, out, ws)
    want = 1.5 * 2.0 ** (byte - 127)
    assert np.abs(out.double().cpu().numpy() / want - 1).max() <= 2.0 ** -20
