"""What the operators over a paged cache refuse, before anything reaches a GPU, their tables of frequencies and sizes (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import page_reference as R  # noqa: E402
from paper_2410_01699_amd import binding as B  # noqa: E402

BAD = B.SJD_EINVAL
P = 1 << 20                 # an address that no refused call touches
ODD = P + 8
MAX = 2 ** 31 - 1


def pool(**change):
    return C.byref(B.sjd_pages(**dict(dict(dtype=0, n_kv_heads=2, head_dim=64, page=32, n_pages=9), **change)))


def call(name, args, **change):
    return getattr(B._lib, name)(*dict(args, **change).values())


TURNS = dict(theta=1e4, rot=64, scaling=0, factor=1.0, original=0.0, slow=1.0, fast=32.0, turns=P)
ROPE = dict(dtype=0, x=P, ldx=128, out=P, ldo=128, pos=P, rows=4, heads=2, hd=64, turns=P, rot=64, inter=0, magnitude=1.0, inverse=0, stream=None)
APPEND = dict(pages=pool(), q=P, ldq=256, heads=4, q_out=P, ldqo=256, k=P, v=P, ld=128, rows=4, start=P, len=P, n_seqs=2, table=P, width=3, turns=P, rot=64, inter=0,
              magnitude=1.0, cache=P, stream=None)
ATTEND = dict(pages=pool(), q=P, ldq=256, heads=4, rows=4, start=P, len=P, n_seqs=2, table=P, width=64, groups=P, prefix=P, n_groups=1, cache=P, scale=0.125, window=0, sinks=0,
              out=P, ldo=256, ws=P, ws_bytes=1 << 40, stream=None)
NORM = dict(dtype=0, x=P, ldx=64, post=P, gate=P, ldg=64, scale=1.0, resid=P, ldr=64, pre=P, eps=1e-5, rows=4, d=64, out=P, ldo=64, stream=None)
POOLS = [dict(pages=None)] + [dict(pages=pool(**c)) for c in (dict(dtype=2), dict(n_kv_heads=0), dict(n_kv_heads=5000), dict(head_dim=80), dict(head_dim=0), dict(page=0),
                                                              dict(page=16), dict(page=48), dict(page=1 << 17), dict(n_pages=0), dict(n_pages=-1))]
SEQS = [dict(start=None), dict(len=None), dict(table=None), dict(rows=0), dict(rows=1 << 25), dict(n_seqs=0), dict(n_seqs=1 << 17), dict(width=0), dict(width=MAX // 32 + 1)]

REFUSED = [
    ("sjd_rope_turns", TURNS, [dict(turns=None), dict(rot=0), dict(rot=3), dict(rot=258), dict(theta=1.0), dict(theta=float("nan")), dict(theta=1e31), dict(scaling=-1),
                               dict(scaling=4), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")), dict(scaling=2, factor=2.0, rot=2), dict(scaling=3, factor=2.0, original=0.0),
                               dict(scaling=3, factor=2.0, original=4096.0, slow=0.0), dict(scaling=3, factor=2.0, original=4096.0, slow=32.0, fast=32.0)]),
    ("sjd_rope", ROPE, [dict(dtype=2), dict(x=None), dict(out=None), dict(pos=None), dict(turns=None), dict(turns=P + 4), dict(ldx=127), dict(ldo=127), dict(rows=0), dict(heads=0), dict(heads=1 << 20),
                        dict(hd=63), dict(hd=0), dict(hd=258), dict(rot=0), dict(rot=63), dict(rot=66), dict(inter=2), dict(magnitude=float("nan")), dict(magnitude=float("inf")),
                        dict(inverse=2), dict(rows=MAX)]),
    ("sjd_page_append", APPEND, POOLS + SEQS + [dict(k=None), dict(v=None), dict(cache=None), dict(cache=ODD), dict(ld=127), dict(q=None), dict(q_out=None), dict(ldq=255), dict(ldqo=255),
                                                dict(heads=0), dict(heads=5000, ldq=1 << 20, ldqo=1 << 20), dict(turns=None), dict(turns=None, rot=0), dict(rot=0), dict(rot=66), dict(rot=63),
                                                dict(inter=-1), dict(magnitude=float("nan"))]),
    ("sjd_page_attention", ATTEND, POOLS + SEQS + [dict(q=None), dict(cache=None), dict(out=None), dict(cache=ODD), dict(ldq=255), dict(ldo=255), dict(heads=3), dict(heads=1), dict(heads=0),
                                                   dict(heads=8192, ldq=1 << 20, ldo=1 << 20), dict(groups=None), dict(prefix=None), dict(n_groups=-1), dict(n_groups=3), dict(scale=0.0),
                                                   dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(sinks=-1), dict(ws=None), dict(ws=ODD),
                                                   dict(ws_bytes=64)]),
    ("sjd_block_norm", NORM, [dict(dtype=2), dict(x=None), dict(resid=None), dict(ldx=63), dict(ldr=63), dict(ldo=63), dict(ldg=63), dict(pre=None), dict(out=None), dict(eps=-1.0),
                              dict(eps=float("nan")), dict(scale=float("nan")), dict(scale=float("inf")), dict(rows=0), dict(rows=MAX), dict(d=0), dict(d=B.SJD_NORM_MAX_D + 1, ldx=1 << 20, ldr=1 << 20, ldg=1 << 20, ldo=1 << 20)]),
]


@pytest.mark.parametrize("name,args,change", [(n, a, c) for n, a, cs in REFUSED for c in cs], ids=lambda v: v if isinstance(v, str) else "-".join(v) if len(v) < 4 else "")
def test_the_entry_refuses(name, args, change):
    assert call(name, args, **change) == BAD


@pytest.mark.parametrize("rot,theta", [(2, 1e4), (20, 1e4), (64, 5e5), (128, 1e4), (256, 1e7)])
@pytest.mark.parametrize("scaling,kw", [(0, {}), (1, dict(factor=4.0)), (2, dict(factor=8.0)), (3, dict(factor=16.0, original=4096.0)), (3, dict(factor=8.0, original=8192.0, slow=1.0, fast=4.0))])
def test_frequencies(rot, theta, scaling, kw):
    """to 2^-48 of each: a power and five roundings in 64 bits"""
    if scaling == 2 and rot == 2:
        return
    t = B.sjd_rope_turns(theta, rot, scaling, **kw)
    want = R.turns(R.frequencies(rot, theta, scaling, **kw)).view(np.uint64).astype(np.float64)
    assert t.dtype == np.int64 and t.shape == (rot // 2,)
    assert (np.abs(t.view(np.uint64).astype(np.float64) - want) <= want * 2.0 ** -48 + 1).all()


def test_a_record_holds_every_value_once():
    for bf16 in (True, False):
        for hd in (32, 96, 256):
            k, v = R.record_at(hd, bf16)
            assert sorted(k.reshape(-1).tolist() + v.reshape(-1).tolist()) == list(range(64 * hd))


def test_workspaces():
    p = B.sjd_pages(1, 8, 128, 64, 1000)
    # short caches that nothing is shared of need none; a workspace does not grow with the cache
    assert B.sjd_page_attention_workspace(p, 4, 4, 0, 32, 16) == 0
    assert B.sjd_page_attention_workspace(p, 4, 4, 0, 32, 17) == B.sjd_page_attention_workspace(p, 4, 4, 0, 32, 1 << 20) > 0
    assert B.sjd_page_attention_workspace(p, 4, 4, 1, 32, 4) > 0
    with pytest.raises(B.SjdError):
        B.sjd_page_attention_workspace(p, 4, 4, 0, 12, 17)
    assert B._lib.sjd_page_attention_workspace(C.byref(p), 4, 4, 0, 32, 16, None) == BAD


def test_the_binding_refuses_what_is_not_on_the_gpu():
    x, i = torch.empty(2, 64), torch.zeros(2, dtype=torch.int32)
    t, p = torch.zeros(32, dtype=torch.int64), B.sjd_pages(0, 1, 64, 32, 1)
    table, cache = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(4096)
    for f in (lambda: B.sjd_rope(x, x, i, 64, t), lambda: B.sjd_page_append(p, x, x, i, i[:1], table, cache),
              lambda: B.sjd_page_attention(p, x, i, i[:1], table, cache, x, None, 0.125), lambda: B.sjd_block_norm(x, x, 1e-5)):
        with pytest.raises(B.SjdError) as e:
            f()
        assert e.value.code == BAD
