"""The operators over a paged cache where sizes and inputs are at their edges (GPU only), against page_reference; tolerances as in test_gpu_page."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import page_reference as R  # noqa: E402
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
