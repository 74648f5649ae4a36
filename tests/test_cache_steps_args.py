"""Windowed and tree attention over the paged cache, its keys' weights, selection and compaction refuse bad arguments
before touching the GPU (these run without one; the pointers are no memory)."""
import pytest

from test_cache_args import ALIGN, ATTEND, BLOCKS, CACHE, L, LONG, NULL, SHAPE, SHARED_BAD, UNSUPPORTED, VALUE, far  # noqa: F401

HEAD = [n for n in ATTEND if n not in ("causal", "max_q", "max_kv", "out", "ost", "ws", "ws_bytes", "stream")]
TAIL = ["max_q", "max_kv", "out", "ost", "ws", "ws_bytes", "stream"]


def call(**middle):
    return dict({n: ATTEND[n] for n in HEAD}, **middle, **{n: ATTEND[n] for n in TAIL})


WINDOW = call(window=100, sinks=4, causal=1)
TREE = call(tree=far(40), words=2)
WEIGHTS = call(before=far(41), after=far(42), causal=1)
ATTEND_BAD = SHARED_BAD + [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(Hq=7), VALUE), (dict(Hq=0), SHAPE), (dict(max_q=-1), SHAPE),
    (dict(max_kv=-1), SHAPE), (dict(qst=1028), ALIGN), (dict(ost=512), SHAPE), (dict(out=far(2) + 8), ALIGN),
    (dict(out=far(1)), SHAPE), (dict(out=far(20) + BLOCKS * 4096 - 16), SHAPE), (dict(Hq=514), VALUE),
]
WINDOW_BAD = ATTEND_BAD + [(dict(window=0), VALUE), (dict(window=-1), VALUE), (dict(sinks=-1), VALUE)]
TREE_BAD = ATTEND_BAD + [
    (dict(tree=None), NULL), (dict(words=0), SHAPE), (dict(words=(1 << 19) + 1), SHAPE), (dict(tree=far(40) + 2), ALIGN),
    (dict(tree=far(2)), SHAPE), (dict(tree=far(2) - 9 * 2 * 4 + 4), SHAPE),
]
WB = 10 * 2 * 64 * 4  # bytes of the weights
WEIGHTS_BAD = ATTEND_BAD + [
    (dict(after=None), NULL), (dict(after=far(42) + 2), ALIGN), (dict(before=far(41) + 1), ALIGN), (dict(after=far(1)), SHAPE),
    (dict(after=far(2) - WB + 4), SHAPE), (dict(before=far(2)), SHAPE), (dict(after=far(21)), SHAPE),
    (dict(before=far(42) + 4), SHAPE), (dict(after=far(41) + WB - 4), SHAPE), (dict(ws=far(42), ws_bytes=1 << 30), SHAPE),
    (dict(ws=far(41) + 16, ws_bytes=1 << 30), SHAPE), (dict(ws=far(30), ws_bytes=16), 10), (dict(ws=far(30) + 8, ws_bytes=1 << 30), ALIGN),
]
CALLS = [("mxattn_cache_attend_window", WINDOW, c) for c in WINDOW_BAD] + [("mxattn_cache_attend_tree", TREE, c) for c in TREE_BAD]
CALLS += [("mxattn_cache_attend_weights", WEIGHTS, c) for c in WEIGHTS_BAD]

BATCH = dict(pages=10, page=64, table=far(11), lens=far(13), seqs=3, max_pages=4)
SELECT = dict(w=far(41), **BATCH, H=2, budget=100, sinks=4, recent=50, kept=far(43), counts=far(44), ws=None, ws_bytes=0, stream=None)
SELECT_BAD = [(dict([(n, None)]), NULL) for n in ("w", "table", "lens", "kept", "counts")] + [
    (dict(pages=0), SHAPE), (dict(page=48), VALUE), (dict(seqs=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(H=0), SHAPE),
    (dict(seqs=1 << 20, H=4), SHAPE), (dict(budget=0), VALUE), (dict(budget=(1 << 24) + 1), VALUE), (dict(sinks=-1), VALUE),
    (dict(recent=-1), VALUE), (dict(sinks=51), VALUE), (dict(sinks=101, recent=0), VALUE), (dict(recent=1 << 62, sinks=1), VALUE),
    (dict(w=far(41) + 2), ALIGN), (dict(kept=far(43) + 2), ALIGN), (dict(counts=far(44) + 1), ALIGN), (dict(lens=far(13) + 2), ALIGN),
    (dict(kept=far(41) + WB - 4), SHAPE), (dict(kept=far(44)), SHAPE), (dict(kept=far(13) - 2400 + 4), SHAPE),
    (dict(counts=far(41)), SHAPE), (dict(counts=far(13) + 8), SHAPE), (dict(kept=far(11)), SHAPE), (dict(counts=far(11) + 44), SHAPE),
]
COMPACT = dict(CACHE, pages=10, page=64, table=far(11), seqs=3, max_pages=4, out=far(45), out_pages=2, H=2, d=128, kept=far(43),
               kept_heads=2, width=100, counts=far(44), base=far(46), w=far(41), stream=None)
COMPACT_BAD = [(dict([(n, None)]), NULL) for n in ("kc", "ks", "vc", "vs", "table", "kept", "counts")] + [
    (dict(pages=0), SHAPE), (dict(page=48), VALUE), (dict(seqs=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(H=0), SHAPE),
    (dict(seqs=1 << 20, H=4), SHAPE), (dict(d=64), UNSUPPORTED), (dict(out_pages=0), SHAPE), (dict(out_pages=1 << 20), SHAPE),
    (dict(kept_heads=3), SHAPE), (dict(kept_heads=0), SHAPE), (dict(width=0), SHAPE), (dict(width=(1 << 24) + 1), SHAPE),
    (dict(kc=far(20) + 8), ALIGN), (dict(kept=far(43) + 2), ALIGN), (dict(base=far(46) + 1), ALIGN), (dict(w=far(41) + 2), ALIGN),
    (dict(out=far(45) + 2), ALIGN), (dict(out=far(11), out_pages=3), SHAPE), (dict(counts=far(44) + 2), ALIGN), (dict(w=far(23)), SHAPE), (dict(w=far(20) - WB + 4), SHAPE),
]
LONG_SELECT = dict(SELECT, page=4096, max_pages=5)
LONG_SELECT_BAD = [
    (dict(ws=far(30), ws_bytes=1000), 10), (dict(ws=far(30) + 8, ws_bytes=1 << 30), ALIGN), (dict(ws=far(41), ws_bytes=1 << 30), SHAPE),
    (dict(ws=far(43) + 2384, ws_bytes=1 << 30), SHAPE), (dict(ws=far(44), ws_bytes=1 << 30), SHAPE),
    (dict(ws=far(13), ws_bytes=1 << 30), SHAPE), (dict(ws=far(11) + 48, ws_bytes=1 << 30), SHAPE),
]
LONG_TREE = dict(TREE, page=4096, max_pages=50, max_q=1)
CALLS += [("mxattn_cache_attend_tree", LONG_TREE, (dict(ws=ws, ws_bytes=1 << 30), SHAPE)) for ws in (far(40), far(40) + 64, far(40) - 16)]
CALLS += [("mxattn_cache_select", LONG_SELECT, c) for c in LONG_SELECT_BAD]
CALLS += [("mxattn_cache_select", SELECT, c) for c in SELECT_BAD] + [("mxattn_cache_compact", COMPACT, c) for c in COMPACT_BAD]


@pytest.mark.parametrize("i", range(len(CALLS)))
def test_refusals(L, i):  # noqa: F811
    name, base, (change, want) = CALLS[i]
    assert getattr(L, name)(*{n: v for n, v in dict(base, **change).items() if n in base}.values()) == want, (name, change)


def test_short_workspaces_are_named_by_their_call(L):  # noqa: F811
    for name, base in (("mxattn_cache_attend_tree", TREE), ("mxattn_cache_attend_weights", WEIGHTS),
                       ("mxattn_cache_attend_window", dict(WINDOW, window=100000))):
        a = dict(base, page=4096, max_pages=50, max_q=1, ws=far(30), ws_bytes=16)
        assert getattr(L, name)(*a.values()) == 10
        detail = L.mxattn_last_error().decode()
        assert name + ":" in detail and "has 16" in detail
    assert "mxattn_cache_attend_weights_workspace" in L.mxattn_status_string(10).decode()


def test_weights_workspace_sizes(L):  # noqa: F811
    size, plain = L.mxattn_cache_attend_weights_workspace, L.mxattn_cache_attend_workspace
    ok = (64, 3, 50, 9, 8, 2, 1, 3200)
    rows = 9 * 8
    assert size(*ok) == (plain(*ok) + 15) // 16 * 16 + rows * 8 + rows * 3200 * 4
    assert size(*ok[:-1], 3190) == size(*ok)  # whole blocks of scores
    assert size(*ok[:-2], 9, 3200) == (plain(*ok[:-2], 9, 3200) + 15) // 16 * 16 + rows * 8  # many rows keep none
    assert size(*ok[:-2], 0, 0) == size(*ok[:-2], 9, 3200)
    long = (4096, 64, 4000, 64, 32, 8, 1, 0)  # scores of 16 M keys would take 134 GB
    assert size(*long) == (plain(*long) + 15) // 16 * 16 + 64 * 32 * 8
    for i, bad in ((0, 48), (1, 0), (2, 0), (3, 0), (4, 7), (5, 0), (6, -1), (7, -1)):
        assert size(*ok[:i], bad, *ok[i + 1:]) == 0, (i, bad)


def test_select_workspace_sizes(L):  # noqa: F811
    size = L.mxattn_cache_select_workspace
    assert size(64, 3, 256, 2) == 0 and size(4096, 3, 4, 2) == 0  # a workgroup holds the keys
    assert size(4096, 1 << 18, 4096, 1) == 0  # more chunks than a launch holds
    assert size(4096, 16, 16, 8) == 0 < size(4096, 16, 17, 8) and 0 < size(4096, 15, 16, 8)  # many heads: of longer ones too
    one = size(64, 1, 257, 1)
    assert 0 < one <= 1.2 * 2 ** 20 and one % 16 == 0 and size(64, 3, 257, 2) == 6 * one
    assert size(4096, 1, 4096, 1) <= 2.3e6
    for bad in ((48, 1, 257, 1), (64, 0, 257, 1), (64, 1, 0, 1), (64, 1, 257, 0), (64, 1 << 20, 257, 4)):
        assert size(*bad) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    """Checks of the Python binding that come before the library; no GPU is needed to fail them."""
    import torch

    from paper_2607_24377_amd import mxattn

    shapes = mxattn.cache_shapes(4, 2, 64)
    cache = [torch.zeros(s, dtype=torch.uint8) for s in shapes]
    table, start, lens = (torch.zeros(s, dtype=torch.int32) for s in ((3, 2), (4,), (3,)))
    q = torch.zeros((5, 2, 128), dtype=torch.bfloat16)
    tree = torch.zeros((5, 1), dtype=torch.int32)
    w = torch.zeros((4, 2, 64))
    with pytest.raises(ValueError):
        mxattn.cache_attend_window(q, *cache, table, start, lens, 10)  # not on a GPU
    with pytest.raises(ValueError):
        mxattn.cache_attend_tree(q, *cache, table, start, lens, tree)
    with pytest.raises(ValueError):
        mxattn.cache_attend_weights(q, *cache, table, start, lens, w)
    with pytest.raises(ValueError):
        mxattn.cache_select(w, table, lens, 10)
    with pytest.raises(ValueError):
        mxattn.cache_compact(*cache, table, torch.zeros((3, 2, 5), dtype=torch.int32), lens)
