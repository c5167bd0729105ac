"""The operators over a paged cache where sizes and inputs are at their edges (GPU only), against page_reference; tolerances as in test_gpu_page."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import page_reference as R  # noqa: E402
import test_gpu_page as G  # noqa: E402
from test_gpu_page import B, Paged, host, ints, own, rnd  # noqa: E402, F401

pytestmark = pytest.mark.gpu


# ---- starts and groups without sense ----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n_seqs,tokens,heads,kv,width,start,groups", [
    (16, 4, 8, 2, 8, "ascending", "again"),             # 8 groups of all sequences: 128 slots of prefixes alone, room for 64 in all
    (60, 3, 8, 2, 40, "again", "again"), (70, 3, 8, 2, 40, "again", "again"), (60, 2, 4, 4, 40, "again", "none"), (151, 2, 8, 1, 40, "again", "again"),
    (4, 160, 64, 8, 40, "again", "again"), (16, 40, 64, 8, 40, "ascending", "again")])
def test_the_join_takes_no_word_of_another_call(B, n_seqs, tokens, heads, kv, width, start, groups, dtype):
    """Starts and groups that repeat ask for more slots than a launch has; the workspace holds words as a call of more rows leaves them, which name rows behind these"""
    c = Paged(B, n_seqs, kv, 64, 32, width, dtype)
    rows, margin = n_seqs * tokens, 16
    starts = [tokens * b for b in range(n_seqs + 1)] if start == "ascending" else [0 if b % 2 == 0 else rows for b in range(n_seqs + 1)]
    bounds = None if groups == "none" else [0 if g % 2 == 0 else n_seqs - 1 for g in range(n_seqs // 2 + 1)]
    n_groups = len(bounds) - 1 if bounds else 0
    word = [rows + margin // 2, margin // 4 * (heads // kv), 0, 0, 2, 0, 0, 0]      # rows that follow, one tile, of two parts
    size = B.sjd_page_attention_workspace(c.pages, rows, n_seqs, n_groups, heads, width)
    q, out = rnd(3, rows, heads * 64).to(c.cache.dtype).cuda(), torch.full((rows + margin, heads * 64), 7.0, dtype=c.cache.dtype, device="cuda")
    ws = ints(word).repeat(size // 32 + 1).view(torch.uint8)[:size].contiguous()
    B.sjd_page_attention(c.pages, q, ints(starts), ints([min(100, 32 * width - rows)] * n_seqs), c.dev(), c.cache, out[:rows], ws, 0.125,
                         groups=ints(bounds) if bounds else None, prefix=ints([96] * n_groups) if bounds else None)
    assert (out[rows:] == 7).all()


# ---- scores at the ends of their range ----------------------------------------------------------------
# (length, tokens, heads, kv heads, width in pages of 32, more): one walk; cut walks; a shared prefix; 128-row tiles in bf16, with edges, cut, and behind a prefix
SHAPES = [([7, 40], [70, 3], 4, 2, 8, {}), ([1200, 3], [2, 1], 4, 2, 42, {}), ([100, 70, 64], [1, 9, 2], 8, 2, 8, dict(groups=[0, 3], prefix=[64])),
          ([900, 950], [1, 2], 8, 2, 40, dict(groups=[0, 2], prefix=[896])), ([0, 300], [320, 129], 64, 8, 26, {}), ([1100], [520], 64, 8, 52, {}),
          ([128, 140], [200, 130], 64, 8, 26, dict(groups=[0, 2], prefix=[128]))]


def filled(B, length, tokens, kv, width, more, hd, dtype, keys):
    """a cache whose positions hold keys(p, k) in place of its random keys k [positions, kv, hd]"""
    c = Paged(B, len(length), kv, hd, 32, width, dtype)
    if more:
        c.table[:, :more["prefix"][0] // 32] = c.table[0, :more["prefix"][0] // 32]
    at, _ = R.record_at(hd, c.bf16)
    ref = c.ref.copy()
    for b in range(len(length)):
        for p in range(length[b] + tokens[b]):
            rec = ref[c.table[b, p // 32], :, 0]
            rec[:, at[p % 32]] = keys(p, rec[:, at[p % 32]])
    c.cache.copy_(torch.from_numpy(ref))
    c.ref = host(c.cache)
    return c


def attended(c, q, length, tokens, heads, scale, more):
    start = np.concatenate(([0], np.cumsum(tokens))).tolist()
    q = torch.from_numpy(q.reshape(len(q), -1)).to(c.cache.dtype).cuda()
    out = torch.full_like(q, 7.0)
    ws = torch.full((c.B.sjd_page_attention_workspace(c.pages, len(q), len(length), len(more.get("prefix", [])), heads, c.table.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda")
    c.B.sjd_page_attention(c.pages, q, ints(start), ints(length), c.dev(), c.cache, out, ws, scale, **{k: ints(v) for k, v in more.items()})
    return host(out).reshape(len(q), heads, c.hd), host(q).reshape(len(q), heads, c.hd)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("length,tokens,heads,kv,width,more", SHAPES)
def test_scores_that_overflow(B, length, tokens, heads, kv, width, more, hd, dtype):
    """Positions below `low` score -2^140, the last one 2^140: rows that see only the former, or the latter, give NaN; to others the former are as good as not there"""
    last = length[0] + tokens[0] - 1
    for low in (length[0] + tokens[0] * 2 // 3, 33, 10 ** 6):
        def keys(p, k):
            k = k.copy()
            k[:, 0] = -2.0 ** 70 if p < low else 2.0 ** 70 if p == last else 0.0
            return k
        c = filled(B, length, tokens, kv, width, more, hd, dtype, keys)
        q = rnd(4, sum(tokens), heads, hd).double().numpy()
        q[..., 0] = 2.0 ** 70
        scale = float(np.float32(1 / np.sqrt(hd)))
        got, q = attended(c, q, length, tokens, heads, scale, more)
        row = 0
        for b, n in enumerate(length):
            k, v, _ = R.sequence(c.ref, c.table[b], 32, n + tokens[b], c.bf16)
            for p in range(n, n + tokens[b]):
                some = [j for j in range(low, p + 1)]
                for h in range(row % 5, heads, 1 if len(got) < 100 else 13):
                    if not some or some[-1] >= last and last >= low:
                        assert np.isnan(got[row, h]).all(), (low, b, p)
                        continue
                    ks, vs = k[some, h // (heads // kv), 1:], v[some, h // (heads // kv)]
                    s = ks @ q[row, h, 1:] * scale
                    w = np.exp(s - s.max())
                    want, top = w @ vs / w.sum(), np.abs(vs).max()
                    d = (hd + 8) * 2.0 ** -24 * (np.abs(ks) @ np.abs(q[row, h, 1:])).max() * scale
                    room = (np.expm1(2 * d) + 2.0 ** -20 + (len(some) / 4 + 64) * 2.0 ** -24 + (2.0 ** -8 if c.bf16 else 0)) * top
                    assert (np.abs(got[row, h] - want) <= room + own(np.abs(want) + room, dtype)).all(), (low, b, p, h)
                row += 1


LN2 = float(np.float32(np.log(2)))              # (times log2 e, in fp32, is 1: a score is then a power of two as the product gives it)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("length,tokens,heads,kv,width,more", SHAPES)
def test_scores_far_off_with_small_differences(B, length, tokens, heads, kv, width, more, hd, dtype):
    """Whole-number scores 2^22 below zero, about it or 2^22 above it, by rows, and for half of the heads 2^21 more from the middle on: all exact in fp32, so weights are as well as near zero"""
    rng = np.random.RandomState(1)
    mid = (length[0] + tokens[0]) // 2

    def keys(p, k):
        k = np.zeros_like(k)
        k[:, 0], k[:, 1] = 2.0 ** 11, 2.0 ** 10 if p >= mid else 0.0
        k[:, 2:10] = rng.randint(-2, 3, (len(k), 8))
        return k
    c = filled(B, length, tokens, kv, width, more, hd, dtype, keys)
    q = np.zeros((sum(tokens), heads, hd))
    q[..., 0] = np.array([-1.0, 0.0, 1.0, 1.0, -1.0])[np.arange(len(q)) * 7 // 3 % 5, None] * 2.0 ** 11
    q[:, ::2, 1] = 2.0 ** 11
    q[..., 2:10] = rng.randint(-1, 2, (len(q), heads, 8))
    got, q = attended(c, q, length, tokens, heads, LN2, more)
    start = np.concatenate(([0], np.cumsum(tokens)))
    want, _, top = R.attention(c.ref, q, start, length, c.table, 32, LN2, c.bf16)
    n = max(x + y for x, y in zip(length, tokens))
    # (differences up to 64 times ln 2's own rounding, below 2^-21)
    room = (2.0 ** -20 + 2.0 ** -21 + (n / 4 + 64) * 2.0 ** -24 + (2.0 ** -8 if c.bf16 else 0)) * top[..., None]
    assert (np.abs(got - want) <= room + own(np.abs(want) + room, dtype)).all(), np.max(np.abs(got - want) / room)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("length,tokens,heads,kv,width,more", SHAPES)
def test_large_values_behind_a_late_reference(B, length, tokens, heads, kv, width, more, dtype):
    """Values up to 2^80 stay finite where later scores are as far above the first ones as a reference may lag, 2^15 in weight"""
    def keys(p, k):
        k = np.zeros_like(k)
        k[:, 0] = 15.0 if p % 64 >= 32 or p > 600 else 0.0
        return k
    c = filled(B, length, tokens, kv, width, more, 64, dtype, keys)
    at = R.record_at(64, c.bf16)[1].reshape(-1)
    c.ref[..., at] *= 2.0 ** 78 / np.abs(c.ref[..., at]).max()
    c.cache.copy_(torch.from_numpy(c.ref))
    c.ref = host(c.cache)
    q = np.zeros((sum(tokens), heads, 64))
    q[..., 0] = 1.0
    got, q = attended(c, q, length, tokens, heads, LN2, more)
    want, _, top = R.attention(c.ref, q, np.concatenate(([0], np.cumsum(tokens))), length, c.table, 32, LN2, c.bf16)
    n = max(x + y for x, y in zip(length, tokens))
    room = (2.0 ** -20 + 2.0 ** -21 + (n / 4 + 64) * 2.0 ** -24 + (2.0 ** -8 if c.bf16 else 0)) * top[..., None]
    assert (np.abs(got - want) <= room + own(np.abs(want) + room, dtype)).all(), np.max(np.abs(got - want) / room)


def test_rows_that_see_nothing_give_zeros(B):
    """all pages of a sequence outside the pool, whatever the first record of the pool holds"""
    for dtype in ("fp32", "bf16"):
        for length, tokens, heads, kv, width, more in SHAPES:
            c = Paged(B, len(length), kv, 64, 32, width, dtype)
            c.table[:] = -1
            c.cache[0] = float("nan")
            got, _ = attended(c, rnd(4, sum(tokens), heads, 64).double().numpy(), length, tokens, heads, 0.125, more)
            assert (got == 0).all()


# ---- every kernel and every variant -------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,hd,rot,pad", [(1201, 33, 128, 128, 16), (2001, 41, 64, 32, 0), (1501, 31, 96, 96, 8), (601, 30, 256, 64, 0), (4100, 65, 16, 16, 0)])
def test_many_rows_are_turned(B, rows, heads, hd, rot, pad, interleaved, dtype):
    """four heads a thread, heads that are no multiple of four: near the definition, and to the bit what a call for each 32 rows (one head a thread) gives"""
    assert rows * heads * (hd // 16) >= 1 << 18 > 32 * heads * (hd // 16)
    G.test_rows_are_turned(B, rows, heads, hd, rot, pad, interleaved, dtype)
    t, turns = G.table_of(B, rot)
    x = rnd(1, rows, heads * hd).to(G.TYPES[dtype]).cuda()
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 911 - 70000
    whole, parts = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    B.sjd_rope(x, whole, pos, hd, turns, interleaved=interleaved, magnitude=1.5)
    for r in range(0, rows, 32):
        B.sjd_rope(x[r:r + 32], parts[r:r + 32], pos[r:r + 32], hd, turns, interleaved=interleaved, magnitude=1.5)
    assert torch.equal(whole, parts)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n_seqs,tokens,kv,hd,page,heads,rot,interleaved,pad", [
    (3, 230, 1, 64, 32, 77, 64, False, 0), (3, 230, 1, 64, 64, 77, 32, True, 16), (3, 230, 1, 64, 32, 76, 10, False, 0), (2, 300, 2, 32, 32, 161, 32, False, 3), (40, 3, 1, 128, 32, 25, 128, True, 0),
    (40, 3, 3, 96, 32, 25, 94, True, 0), (40, 2, 1, 256, 32, 27, 256, False, 0), (40, 2, 1, 256, 64, 27, 254, False, 0), (2, 500, 8, 128, 64, 107, 64, False, 0)])
def test_append_with_many_heads(B, n_seqs, tokens, kv, hd, page, heads, rot, interleaved, pad, dtype):
    """two query heads a workgroup, odd numbers of them, by units and by values; ragged tokens"""
    lengths = [(b * 37) % 50 for b in range(n_seqs)]
    counts = [max(0, tokens - b % 3) for b in range(n_seqs)]
    assert (sum(counts) // 32 + 2 * n_seqs) * heads >= 2048
    c = Paged(B, n_seqs, kv, hd, page, -(-(tokens + 60) // page), dtype)
    t = B.sjd_rope_turns(10000.0, rot)
    c.append(lengths, counts, seed=1, heads=heads, t=t, interleaved=interleaved, pad=pad, behind=2)
    lengths[1] = -1                                 # sits out
    c.append(lengths, counts, seed=2, heads=heads, t=t, interleaved=interleaved, magnitude=1.2, pad=pad, inplace=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("length,tokens,heads,kv,kw", [
    ([0, 700], [300, 100], 32, 8, {}), ([0, 700], [300, 100], 32, 8, dict(window=90, sinks=40)), ([20, 31], [150, 263], 32, 8, dict(pad=1)), ([160, 130, 128], [1, 9, 2], 8, 2, dict(groups=[0, 3], prefix=[128])),
    ([800, 810, -1, 790], [3, 9, 2, 20], 16, 2, dict(groups=[0, 4], prefix=[770]))])
def test_tiles_of_32_rows(B, length, tokens, heads, kv, kw, hd, dtype):
    c = Paged(B, len(length), kv, hd, 32, 27, dtype)
    if "prefix" in kw:
        c.table[:, :kw["prefix"][0] // 32] = c.table[0, :kw["prefix"][0] // 32]
    assert "prefix" in kw or (sum(tokens) * heads // kv >> 5) * kv >= 384
    c.check(length, tokens, heads, **kw)


@pytest.mark.parametrize("hd", [32, 64, 96, 128])
@pytest.mark.parametrize("length,tokens,kw", [([1100], [520], {}), ([900, 40], [290, 240], {}), ([1000, 1000], [260, 260], dict(groups=[0, 2], prefix=[992])), ([1100], [520], dict(window=200, sinks=50)),
                                              ([1030, 1100, 1024], [100, 257, 170], dict(groups=[1, 3], prefix=[512]))])
def test_tiles_of_many_rows_over_cut_walks(B, length, tokens, kw, hd):
    c = Paged(B, len(length), 8, hd, 32, 52, "bf16")
    if "prefix" in kw:
        first, last = kw["groups"]
        c.table[first:last, :kw["prefix"][0] // 32] = c.table[first, :kw["prefix"][0] // 32]
    own_tiles = (sum(tokens) * 8 >> 7) + len(length)
    assert (sum(tokens) * 8 >> 7) * 8 >= 256 and own_tiles * 8 < 320
    assert B.sjd_page_attention_workspace(c.pages, sum(tokens), len(length), 0, 64, 52) > 0           # walks are cut
    c.check(length, tokens, 64, **kw)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [32, 96, 128, 256])
@pytest.mark.parametrize("length,tokens,heads,kv,window,sinks", [([1300], [1], 4, 4, 0, 0), ([1500, 3, 700, 1100], [1, 1, 2, 16], 4, 2, 0, 0), ([1500, 40, 1030], [5, 60, 1], 4, 2, 33, 40), ([1023, 1024, 1025], [1, 1, 1], 8, 1, 0, 0)])
def test_cut_walks_of_all_heads(B, length, tokens, heads, kv, window, sinks, hd, dtype):
    Paged(B, len(length), kv, hd, 64, 26, dtype).check(length, tokens, heads, window, sinks)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_seqs,width", [(65, 5), (90, 34)])
def test_tiles_of_many_rows_of_more_sequences_than_lanes(B, n_seqs, width, hd):
    c = Paged(B, n_seqs, 8, hd, 32, width, "bf16")
    groups, prefix = [2, 40, n_seqs - 1], [96, 64]
    for g, p in enumerate(prefix):
        c.table[groups[g]:groups[g + 1], :p // 32] = c.table[groups[g], :p // 32]
    length, tokens = [96 + (b * 7) % 20 for b in range(n_seqs)], [20 - b % 4 for b in range(n_seqs)]
    length[5] = -1
    assert sum(tokens) * 8 // n_seqs >= 64 and (sum(tokens) * 8 >> 7) * 8 >= 256
    c.check(length, tokens, 64, groups=groups, prefix=prefix)
    c.check(length, tokens, 64, behind=3)


def test_a_pool_of_no_dimensions_is_refused(B):
    x, i, cache = torch.zeros(2, 64, device="cuda"), ints([0, 2]), torch.zeros(0, device="cuda")
    for hd in (0, -64):
        p = B.sjd_pages(0, 1, hd, 32, 1)
        for f in (lambda: B.sjd_page_attention(p, x, i, i[1:], i[:1].view(1, 1), cache, x, None, 1.0),
                  lambda: B.sjd_page_append(p, x[:, :0], x[:, :0], i, i[1:], i[:1].view(1, 1), cache, q=x, q_out=x)):
            with pytest.raises(B.SjdError) as e:
                f()
            assert e.value.code == B.SJD_EINVAL


# ---- calls that the header allows ----------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("length,tokens,heads,kv,width,more", SHAPES)
def test_what_masks_hide_of_the_keys(B, length, tokens, heads, kv, width, more, dtype):
    """NaN and infinities in keys behind the last token, to the bit; in a key of the last token of a sequence: that row alone"""
    c = filled(B, length, tokens, kv, width, more, 64, dtype, lambda p, k: k)
    q = rnd(4, sum(tokens), heads, 64).double().numpy()
    clean, _ = attended(c, q, length, tokens, heads, 0.125, more)
    at, _ = R.record_at(64, c.bf16)
    at = torch.from_numpy(at).cuda()
    for b, n in enumerate(length):
        end = n + tokens[b]
        for p in range(end, (end + 31) // 32 * 32):
            c.cache[c.table[b, p // 32]][:, 0, at[p % 32]] = float("nan") if p % 2 else float("inf")
    got, _ = attended(c, q, length, tokens, heads, 0.125, more)
    assert np.array_equal(got, clean)
    row = 0
    for b, n in enumerate(length):
        row += tokens[b]
        p = n + tokens[b] - 1
        c.cache[c.table[b, p // 32]][:, 0, at[p % 32, 5]] = float("nan")
        clean[row - 1] = np.nan
    got, _ = attended(c, q, length, tokens, heads, 0.125, more)
    assert np.array_equal(got, clean, equal_nan=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("length,tokens,heads,kv,width,more", SHAPES)
def test_a_query_that_is_not_finite_stays_alone(B, length, tokens, heads, kv, width, more, dtype):
    c = filled(B, length, tokens, kv, width, more, 64, dtype, lambda p, k: k)
    q = rnd(4, sum(tokens), heads, 64).double().numpy()
    clean, _ = attended(c, q, length, tokens, heads, 0.125, more)
    q[1, 1, 3], q[len(q) - 1, heads - 1, 60] = np.nan, np.nan
    got, _ = attended(c, q, length, tokens, heads, 0.125, more)
    clean[1, 1] = clean[len(q) - 1, heads - 1] = np.nan
    assert np.array_equal(got, clean, equal_nan=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("length,tokens,heads,kv,width,more", SHAPES)
def test_rows_before_the_first_sequence(B, length, tokens, heads, kv, width, more, dtype):
    """starts from 5 on give the same bits five rows further on, and leave the rows before them"""
    c = filled(B, length, tokens, kv, width, more, 64, dtype, lambda p, k: k)
    rows, start = sum(tokens), np.concatenate(([0], np.cumsum(tokens)))
    x = rnd(4, rows + 5, (heads + 2 * kv) * 64).to(c.cache.dtype).cuda()
    q, k, v = x[:, :heads * 64], x[:, heads * 64:(heads + kv) * 64], x[:, (heads + kv) * 64:]
    turns = torch.from_numpy(B.sjd_rope_turns(10000.0, 64)).cuda()
    ws = torch.full((B.sjd_page_attention_workspace(c.pages, rows + 5, len(length), len(more.get("prefix", [])), heads, width),), 0xFF, dtype=torch.uint8, device="cuda")
    results = []
    for shift in (5, 0):
        cache, part = c.cache.clone(), slice(5 - shift, None)
        turned, out = (torch.full((rows + shift, heads * 64), 7.0, dtype=x.dtype, device="cuda") for _ in range(2))
        s, n, table = ints((start + shift).tolist()), ints(length), c.dev()
        B.sjd_page_append(c.pages, k[part], v[part], s, n, table, cache, turns=turns, q=q[part], q_out=turned)
        B.sjd_page_attention(c.pages, turned, s, n, table, cache, out, ws, 0.125, **{key: ints(y) for key, y in more.items()})
        assert (turned[:shift] == 7).all() and (out[:shift] == 7).all()
        results.append((cache, turned[shift:], out[shift:]))
    # (five rows more can choose other tiles: each result is off by at most 2^-8 + 2^-8 (bf16), 2^-12 (fp32: scores up to 15 off by 72 roundings, 470 of sums) of the largest value)
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    assert (results[0][2].double() - results[1][2].double()).abs().max() <= (2.0 ** -6 if c.bf16 else 2.0 ** -11) * c.cache.double().abs().max()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("page,length,tokens", [(1024, [1000, 2040], [40, 9]), (65536, [1030, 0], [3, 33]), (65536, [65530, 65536 + 31], [9, 2])])
def test_long_pages(B, page, length, tokens, dtype):
    c = Paged(B, 2, 2, 32, page, 3 if page == 1024 else 2, dtype, spare=1)
    c.append(length, tokens, heads=2, t=B.sjd_rope_turns(10000.0, 32))
    c.check(length, tokens, 4)
    c.check(length, tokens, 4, window=700, sinks=5)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,kv,tokens", [(4096, 1, [2, 1]), (4096, 4096, [1, 2]), (4095, 4095, [1, 0]), (999, 333, [3, 1])])
def test_as_many_heads_as_there_may_be(B, heads, kv, tokens, dtype):
    c = Paged(B, 2, kv, 32, 32, 2, dtype)
    c.append([30, 5], tokens, heads=heads, t=B.sjd_rope_turns(10000.0, 32))
    c.check([30, 5], tokens, heads)
