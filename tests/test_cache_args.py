"""The entry points of the norm and rotation and of the paged cache refuse bad arguments before touching the GPU
(these run without one; the pointers are no memory)."""
import ctypes
import os

import pytest

FAKE = 0x100000
NULL, SHAPE, ALIGN, UNSUPPORTED, VALUE = 1, 2, 3, 6, 11


@pytest.fixture(scope="module")
def L():
    from paper_2607_24377_amd import mxattn

    if not os.path.exists(mxattn.LIB_PATH):
        from paper_2607_24377_amd import build

        build.build()
    return mxattn.lib()


def far(i):
    return FAKE + (i << 40)


ROPE = dict(q=far(1), k=far(2), qo=far(3), ko=far(4), B=2, Hq=4, Hkv=2, N=8, d=128, qs=None, ks=None, qos=None, kos=None,
            qw=far(5), kw=far(6), eps=1e-6, cos=far(7), sin=far(8), pos=far(9), rows=100, rot=128, pairs=1, stream=None)
# a bad d is looked at after everything below but the shapes, so each case sets it only where nothing else is wrong
ROPE_BAD = [
    (dict(q=None), NULL), (dict(qo=None), NULL), (dict(k=None), NULL), (dict(ko=None), NULL), (dict(cos=None), NULL),
    (dict(sin=None), NULL), (dict(B=0), SHAPE), (dict(Hq=0), SHAPE), (dict(Hkv=-1), SHAPE), (dict(N=0), SHAPE),
    (dict(d=64), UNSUPPORTED), (dict(rot=8), VALUE), (dict(rot=-16), VALUE), (dict(rot=144), VALUE), (dict(rot=24), VALUE),
    (dict(pairs=2), VALUE), (dict(pairs=-1), VALUE), (dict(eps=-1e-6), VALUE), (dict(eps=float("nan")), VALUE),
    (dict(eps=float("inf")), VALUE), (dict(rows=0), SHAPE), (dict(q=far(1) + 8), ALIGN), (dict(ko=far(4) + 2), ALIGN),
    (dict(qw=far(5) + 4), ALIGN), (dict(cos=far(7) + 4), ALIGN), (dict(pos=far(9) + 2), ALIGN),
    (dict(qs=(4096, 1024, 12)), ALIGN), (dict(qs=(4096, -1024, 128)), SHAPE),
    (dict(qos=(4096, 1024, 0)), SHAPE),      # output rows on one another
    (dict(qos=(4096, 128, 128)), SHAPE), (dict(qos=(2048, 1024, 128)), SHAPE), (dict(kos=(0, 1024, 128)), SHAPE),
    (dict(qo=far(1)), SHAPE),                 # in place
    (dict(qo=far(2) + 2 * 2 * 8 * 256 - 16), SHAPE), (dict(ko=far(3) + 16), SHAPE), (dict(ko=far(1) + 2 * 4 * 8 * 256 - 16), SHAPE),
]


@pytest.mark.parametrize("i", range(len(ROPE_BAD)))
def test_rope_refusals(L, i):
    change, want = ROPE_BAD[i]
    a = dict(ROPE, **change)
    for s in ("qs", "ks", "qos", "kos"):
        if a[s] is not None:
            a[s] = (ctypes.c_int64 * 3)(*a[s])
    assert L.mxattn_qk_norm_rope(*a.values()) == want, change


BATCH = dict(pages=10, page=64, table=far(11), start=far(12), lens=far(13), seqs=3, max_pages=4)
CACHE = dict(kc=far(20), ks=far(21), vc=far(22), vs=far(23))
APPEND = dict(k=far(1), v=far(2), kst=512, vst=512, **CACHE, **BATCH, tokens=9, H=2, d=128, w=far(3), eps=1e-6, cos=far(4),
              sin=far(5), pos=far(6), rows=100, rot=128, pairs=0, stream=None)
SHARED_BAD = [(dict([(n, None)]), NULL) for n in ("kc", "ks", "vc", "vs", "table", "start", "lens")] + [
    (dict(pages=0), SHAPE), (dict(pages=(1 << 30) + 1), SHAPE), (dict(page=0), VALUE), (dict(page=16), VALUE),
    (dict(page=96), VALUE), (dict(page=8192), VALUE), (dict(seqs=0), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(max_pages=(1 << 24) + 1), SHAPE), (dict(tokens=0), SHAPE), (dict(d=64), UNSUPPORTED), (dict(kc=far(20) + 8), ALIGN),
    (dict(vc=far(22) + 8), ALIGN), (dict(table=far(11) + 2), ALIGN), (dict(lens=far(13) + 1), ALIGN),
]
BLOCKS = 10 * 2 * 2
APPEND_BAD = SHARED_BAD + [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(H=0), SHAPE), (dict(H=70000, tokens=1), SHAPE), (dict(kst=-8), SHAPE), (dict(vst=260), ALIGN),
    (dict(k=far(1) + 4), ALIGN), (dict(rot=20), VALUE), (dict(pairs=5), VALUE), (dict(eps=-1.0), VALUE), (dict(cos=None), NULL),
    (dict(k=far(20) + BLOCKS * 4096 - 16), SHAPE), (dict(v=far(23)), SHAPE), (dict(v=far(21) - 8704 + 16), SHAPE),
]


@pytest.mark.parametrize("i", range(len(APPEND_BAD)))
def test_append_refusals(L, i):
    change, want = APPEND_BAD[i]
    assert L.mxattn_cache_append(*dict(APPEND, **change).values()) == want, change


ATTEND = dict(q=far(1), qst=1024, **CACHE, **BATCH, tokens=9, Hq=8, Hkv=2, d=128, causal=1, max_q=0, max_kv=0, out=far(2),
              ost=1024, ws=None, ws_bytes=0, stream=None)
ATTEND_BAD = SHARED_BAD + [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(Hq=7), VALUE), (dict(Hq=0), SHAPE), (dict(Hq=1), VALUE),
    (dict(max_q=-1), SHAPE), (dict(max_kv=-1), SHAPE), (dict(qst=1028), ALIGN), (dict(qst=-1024), SHAPE),
    (dict(ost=512), SHAPE), (dict(out=far(2) + 8), ALIGN), (dict(out=far(1)), SHAPE), (dict(out=far(1) + 9 * 2048 - 16), SHAPE),
    (dict(out=far(20) + BLOCKS * 4096 - 16), SHAPE), (dict(out=far(23) + 16), SHAPE),
]


@pytest.mark.parametrize("i", range(len(ATTEND_BAD)))
def test_attend_refusals(L, i):
    change, want = ATTEND_BAD[i]
    assert L.mxattn_cache_attend(*dict(ATTEND, **change).values()) == want, change


# sizes that the kernels' numbers cannot hold, and workspaces that do not do (of 3 sequences with up to 200000 keys)
LONG = dict(ATTEND, page=4096, max_pages=50, max_q=1)
BIG = [
    ("rope", dict(Hq=65536, B=1, N=1), SHAPE), ("rope", dict(Hkv=65536, B=1, N=1), SHAPE),
    ("append", dict(seqs=(1 << 20) + 1), SHAPE), ("append", dict(page=4096, max_pages=4097), SHAPE),
    ("append", dict(pages=1 << 30, page=4096, H=65535, tokens=1), SHAPE),
    ("attend", dict(Hq=514), VALUE), ("attend", dict(H=65536, Hkv=65536, Hq=65536, tokens=1), SHAPE),
    ("attend", dict(seqs=1 << 20, Hkv=16, Hq=16, tokens=1, qst=2048, ost=2048), SHAPE),
    ("attend", dict(seqs=1 << 20, Hkv=4096, Hq=4096, tokens=1, ost=1 << 19, qst=1 << 19), SHAPE),
    ("long", dict(ws=far(30), ws_bytes=1000), 10), ("long", dict(ws=far(30) + 8, ws_bytes=1 << 30), ALIGN),
    ("long", dict(ws=far(1), ws_bytes=1 << 30), SHAPE), ("long", dict(ws=far(2) - 4096, ws_bytes=1 << 30), SHAPE),
    ("long", dict(ws=far(21), ws_bytes=1 << 30), SHAPE),
]


@pytest.mark.parametrize("i", range(len(BIG)))
def test_sizes_and_workspaces_refused(L, i):
    what, change, want = BIG[i]
    call, base = {"rope": (L.mxattn_qk_norm_rope, ROPE), "append": (L.mxattn_cache_append, APPEND),
                  "attend": (L.mxattn_cache_attend, ATTEND), "long": (L.mxattn_cache_attend, LONG)}[what]
    assert call(*{k: v for k, v in dict(base, **change).items() if k in base}.values()) == want, change


def test_workspace_sizes(L):
    size = L.mxattn_cache_attend_workspace
    ok = (64, 3, 50, 9, 8, 2, 1, 3200)
    assert 0 < size(*ok) <= 65 * 2 ** 20 + 8 * 2 * (3 + 2)
    assert size(*ok[:-1], 1024) == 0 and size(*ok[:3], 90, *ok[4:6], 40, 1024) > 0
    assert size(*ok[:-2], 0, 0) == size(*ok[:-2], 9, 3200)  # 0: whatever the sizes allow
    for i, bad in ((0, 48), (1, 0), (2, 0), (3, 0), (4, 7), (5, 0), (5, 3), (6, -1), (7, -1), (2, 1 << 20)):
        assert size(*ok[:i], bad, *ok[i + 1:]) == 0, (i, bad)


def test_binding_refuses_tensors_that_do_not_fit():
    """Checks of the Python binding that come before the library; no GPU is needed to fail them."""
    import torch

    from paper_2607_24377_amd import mxattn

    x = torch.zeros((1, 2, 3, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mxattn.qk_norm_rope(x, x)  # not on a GPU
    shapes = mxattn.cache_shapes(4, 2, 64)
    assert shapes == ((4, 2, 2, 8, 32, 16), (4, 2, 2), (4, 2, 2, 128, 32), (4, 2, 2))
    cache = [torch.zeros(s, dtype=torch.uint8) for s in shapes]
    table, start, lens = (torch.zeros(s, dtype=torch.int32) for s in ((3, 2), (4,), (3,)))
    q = torch.zeros((5, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mxattn.cache_attend(q, *cache, table, start, lens)  # not on a GPU
    for i, bad in ((0, cache[0][:, :1]), (1, cache[1].int()), (2, cache[2].transpose(3, 4)), (3, cache[3][:2])):
        with pytest.raises(ValueError):
            mxattn.cache_append(q, q, *cache[:i], bad, *cache[i + 1:], table, start, lens)
    for args in ((table.long(), start, lens), (table, start[:3], lens), (table, start, lens[:2]), (table[0], start, lens)):
        with pytest.raises(ValueError):
            mxattn.cache_append(q, q, *cache, *args)
    with pytest.raises(ValueError):
        mxattn.cache_append(q, q[:, :1], *cache, table, start, lens)
