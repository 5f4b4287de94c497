"""What the calls of the paged cache refuse, decided on the host: nothing is launched (no GPU)."""
import ctypes as C

import pytest

from paper_2410_01485_b200 import binding as lg, build

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    build.build()
    return lg.load_library()


def _good(**kw):
    a = dict(B=2, Hq=8, Hkv=2, D=128, sink_tokens=64, window_tokens=256, page_tokens=32, num_pages=40)
    a.update(kw)
    return lg.paged_params(**a)


def _calls(lib, p, **kw):
    """Every entry point on fake, aligned pointers (256), with the named arguments replaced."""
    big = 1 << 40
    n = (C.c_int64 * 4)(10, 10, 10, 10)
    args = {"lg_paged_table_extend": dict(n=256, new=256, T=4, free=256, n_free=9, start=256, table=256, next=512, stream=None),
            "lg_paged_slot_map": dict(n=256, first=256, count=256, T=4, table=256, map=256, stream=None),
            "lg_paged_append": dict(k=256, v=512, ks=256, vs=512, table=256, kn=256, vn=256, strides=None, T=4, n=256, new=256, stream=None),
            "lg_paged_gather": dict(k=256, v=256, ks=256, vs=256, map=256, T=4, ko=256, vo=256, stream=None),
            "lg_paged_decode": dict(q=256, k=256, v=256, ks=256, vs=256, table=256, n=256, o=256, lse=256, ws=256, bytes=big, stream=None),
            "lg_paged_chunk_prefill": dict(q=256, kn=256, vn=256, k=256, v=256, ks=256, vs=256, table=256, T=4, hn=n, o=256, lse=256,
                                           ws=256, bytes=big, stream=None)}
    out = {}
    for name, a in args.items():
        if kw and not any(x in a for x in kw):
            continue
        a = {x: kw.get(x, y) for x, y in a.items()}
        out[name] = getattr(lib, name)(C.byref(p) if p is not None else None, *a.values())
    return out


@pytest.mark.parametrize("change, code", [
    (dict(B=0), INVALID), (dict(Hkv=3), INVALID), (dict(Hq=0), INVALID), (dict(sink_tokens=-1), INVALID), (dict(window_tokens=0), INVALID),
    (dict(page_tokens=0), INVALID), (dict(page_tokens=48), INVALID), (dict(page_tokens=256), INVALID), (dict(num_pages=0), INVALID),
    (dict(table_stride=9), INVALID), (dict(table_stride=-1), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(block_tokens=-1), INVALID), (dict(block_tokens=48), INVALID),
    (dict(D=96), UNSUPPORTED), (dict(num_pages=1 << 25), UNSUPPORTED), (dict(window_tokens=1 << 30), UNSUPPORTED),
])
def test_bad_parameters(lib, change, code):
    p = _good(**change)
    assert set(_calls(lib, p).values()) == {code}
    assert lib.lg_paged_decode_workspace_bytes(C.byref(p)) == 0
    assert lib.lg_paged_chunk_prefill_workspace_bytes(C.byref(p), 4, (C.c_int64 * 2)(1, 1)) == 0


def test_null_parameters(lib):
    assert set(_calls(lib, None).values()) == {INVALID}
    assert lib.lg_paged_decode_workspace_bytes(None) == 0


@pytest.mark.parametrize("arg, bad", [
    ("n", (None, 260)), ("table", (None, 258)), ("free", (None, 258)), ("start", (None, 258)), ("next", (None, 514)), ("first", (None, 260)),
    ("map", (None, 260)), ("k", (None, 264)), ("v", (None, 264)), ("ks", (None, 258)), ("vs", (None, 258)), ("kn", (None, 264)),
    ("vn", (None, 264)), ("ko", (None, 264)), ("vo", (None, 264)), ("q", (None, 264)), ("o", (None, 264)), ("ws", (None, 128)),
    ("new", (258,)), ("count", (258,)), ("lse", (258,)), ("hn", (None,)), ("T", (-1,)), ("n_free", (-1,)),
])
def test_bad_pointers_and_counts(lib, arg, bad):
    for x in bad:
        got = _calls(lib, _good(), **{arg: x})
        assert got and set(got.values()) == {INVALID}, (arg, x, got)


def test_free_start_and_next_are_two_places(lib):
    assert _calls(lib, _good(), next=256)["lg_paged_table_extend"] == INVALID


@pytest.mark.parametrize("strides", [(0, 64, 128), (8192, 1024, 100), (8192, 1024, 64), (-8, 1024, 128), (8192, 1028, 128)])
def test_bad_strides(lib, strides):
    assert _calls(lib, _good(), strides=(C.c_int64 * 3)(*strides))["lg_paged_append"] == INVALID


def test_nothing_to_do_is_no_error(lib):
    got = _calls(lib, _good(), T=0)
    assert got["lg_paged_append"] == got["lg_paged_gather"] == got["lg_paged_slot_map"] == 0


def test_workspaces(lib):
    p = _good()
    need = lib.lg_paged_decode_workspace_bytes(C.byref(p))
    assert need > 256
    assert _calls(lib, p, bytes=need - 1)["lg_paged_decode"] == WORKSPACE
    size = lambda T, *n: lib.lg_paged_chunk_prefill_workspace_bytes(C.byref(_good(B=len(n))), T, (C.c_int64 * len(n))(*n))
    need = size(50, 1000, 7)
    assert _calls(lib, p, hn=(C.c_int64 * 2)(1000, 7), T=50, bytes=need - 1)["lg_paged_chunk_prefill"] == WORKSPACE
    # sequences at any positions are one run, as large as one of full rings
    assert need == size(50, 1000, 2000) > size(50, 1000)
    # but for a sink that is not full under a chunk longer than the window (256): runs of what holds equally many share the space
    assert size(257, 1000, 7) == max(size(257, 1000), size(257, 7)) and size(257, 1000, 70) > size(257, 1000)
    # and for chunks of more than 64 super-tiles
    assert size(17000, 1000, 70) == max(size(17000, 1000), size(17000, 70))


def test_chunk_limits(lib):
    n = (C.c_int64 * 2)(5, 5)
    size = lib.lg_paged_chunk_prefill_workspace_bytes
    assert size(C.byref(_good()), 4, n) > 0
    assert size(C.byref(_good()), 0, n) == 0 and size(C.byref(_good()), 4, (C.c_int64 * 2)(5, -1)) == 0 and size(C.byref(_good()), 4, None) == 0
    assert _calls(lib, _good(sink_tokens=32), T=4)["lg_paged_chunk_prefill"] == UNSUPPORTED
    assert _calls(lib, _good(window_tokens=100), T=4)["lg_paged_chunk_prefill"] == UNSUPPORTED
    assert _calls(lib, _good(), hn=(C.c_int64 * 2)(5, -1))["lg_paged_chunk_prefill"] == INVALID


def test_status_string(lib):
    assert "page" in lg.status_string(-7)


def test_sizes_beyond_what_is_covered(lib):
    assert _calls(lib, _good(), T=(1 << 30) + 1)["lg_paged_slot_map"] == UNSUPPORTED
    assert _calls(lib, _good(B=65536), T=4)["lg_paged_slot_map"] == UNSUPPORTED
    assert _calls(lib, _good(B=65536), T=4)["lg_paged_gather"] == UNSUPPORTED
    assert _calls(lib, _good(B=1 << 30, window_tokens=1 << 20), T=1 << 20)["lg_paged_append"] == UNSUPPORTED
    # one sequence of more tiles than the decode counts
    long = _good(B=1, Hq=256, Hkv=256, window_tokens=(1 << 30) - 64, num_pages=10)
    assert lib.lg_paged_decode_workspace_bytes(C.byref(long)) == 0
    assert _calls(lib, long)["lg_paged_decode"] == UNSUPPORTED


def test_append_writes_two_arrays(lib):
    assert _calls(lib, _good(), v=256)["lg_paged_append"] == INVALID and _calls(lib, _good(), vs=256)["lg_paged_append"] == INVALID
