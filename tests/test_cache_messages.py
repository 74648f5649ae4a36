"""What the cache's calls say when they refuse: the status text and the detail name the call's own cause (no GPU)."""
from test_cache_args import LONG, L, far  # noqa: F401


def test_short_workspace_is_named_with_both_sizes(L):  # noqa: F811
    need = L.mxattn_cache_attend_workspace(4096, 3, 50, 9, 8, 2, 1, 0)
    assert need > 1000
    assert L.mxattn_cache_attend(*dict(LONG, ws=far(30), ws_bytes=1000).values()) == 10
    detail = L.mxattn_last_error().decode()
    assert "mxattn_cache_attend" in detail and str(need) in detail and "1000" in detail


def test_status_text_covers_the_cache(L):  # noqa: F811
    text = L.mxattn_status_string(10).decode()
    assert "mxattn_cache_attend_workspace" in text and "capture" in text and "32768" in text
    assert "stride" in L.mxattn_status_string(3).decode()


def test_the_binding_passes_both_on(L):  # noqa: F811
    from paper_2607_24377_amd import mxattn

    assert L.mxattn_cache_attend(*dict(LONG, ws=far(30), ws_bytes=1000).values()) == 10
    e = mxattn.MxattnError(10, "mxattn_cache_attend")
    assert "workspace" in str(e) and "1000" in str(e)


def test_a_status_without_detail_does_not_show_an_earlier_one(L):  # noqa: F811
    from paper_2607_24377_amd import mxattn

    assert L.mxattn_cache_attend(*dict(LONG, ws=far(30), ws_bytes=1000).values()) == 10
    assert L.mxattn_cache_attend(*dict(LONG, tokens=0).values()) == 2
    assert "workspace needed" not in str(mxattn.MxattnError(2, "mxattn_cache_attend"))
