"""The Python binding's own checks of a paged cache's arrays, on host tensors (`_cache` compares a tensor's device
with the index it is given; -1 is the host)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_24377_amd import mxattn  # noqa: E402

PAGES, HEADS, PAGE, SEQS = 4, 2, 64, 3


def arrays(shapes):
    return [torch.zeros(s, dtype=torch.uint8) for s in shapes]


def batch():
    return [torch.zeros(s, dtype=torch.int32) for s in ((SEQS, 2), (SEQS + 1,), (SEQS,))]


def checked(cache):
    return mxattn._cache(*cache, *batch(), -1, 128)


def test_arrays_of_cache_shapes_are_taken():
    cache = arrays(mxattn.cache_shapes(PAGES, HEADS, PAGE))
    args, heads = checked(cache)
    assert heads == HEADS and args[4:6] == (PAGES, PAGE)
    assert args[:4] == tuple(c.data_ptr() for c in cache)


# the kernels address 4096 bytes of codes for every scale, in this order of the axes
N = PAGE // 32
LEAD = (PAGES, HEADS, N)
BAD = [
    (0, LEAD + (4, 32, 16)),      # 64 channels: half of the bytes
    (0, LEAD + (16, 32, 16)),
    (0, LEAD + (8, 16, 32)),      # as many bytes in another order
    (0, LEAD + (8, 512, 1)),
    (0, (PAGES, HEADS, N, 4096)),
    (2, LEAD + (64, 32)),
    (2, LEAD + (32, 128)),
    (2, (HEADS, PAGES, N, 128, 32)),
    (2, (PAGES * HEADS * N * 4096,)),
]


@pytest.mark.parametrize("i", range(len(BAD)))
def test_codes_of_another_shape_are_refused(i):
    which, shape = BAD[i]
    cache = arrays(mxattn.cache_shapes(PAGES, HEADS, PAGE))
    cache[which] = torch.zeros(shape, dtype=torch.uint8)
    with pytest.raises(ValueError):
        checked(cache)


def test_codes_of_64_channels_are_refused_for_rows_of_128():
    """Both code arrays of half the size, which agree with each other."""
    cache = arrays([LEAD + (4, 32, 16), LEAD, LEAD + (64, 32), LEAD])
    with pytest.raises(ValueError):
        checked(cache)


@pytest.mark.parametrize("page,d", [(64, 64), (64, 256), (48, 128), (16, 128), (8192, 128), (0, 128)])
def test_shapes_that_no_call_takes_are_refused(page, d):
    with pytest.raises(ValueError):
        mxattn.cache_shapes(PAGES, HEADS, page, d)


def test_stream_without_torchs_private_call(monkeypatch):
    """The current stream comes from the public interface where torch has no other."""
    class Stream:
        cuda_stream = 42

    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: Stream if index == 3 else None)
    assert mxattn._raw_stream(3) == 42
