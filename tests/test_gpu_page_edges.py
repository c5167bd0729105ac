"""The operators over a paged cache where sizes and inputs are at their edges (GPU only), against page_reference; tolerances as in test_gpu_page."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_page import B, Paged, ints, rnd  # noqa: E402, F401

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
