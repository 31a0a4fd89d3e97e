"""The page calls without a GPU: one memory for two of a call's arrays, or for an array and the contents
that it moves, is refused before a launch."""

import pytest
import torch

import paper_2609_32197_amd as sp
from paper_2609_32197_amd.bounded import _BUFFER, _PAGES

AT = 1 << 20  # addresses that no refused call touches, this far apart
PAGES, PAGE, WIDTH, B = 900, 16, 40, 30
ROWS = 50  # of a fork

# Of each call: what it takes, in order, the bytes of each and whether the call writes it.
SIZE = {"refs": 4 * PAGES, "table": 4 * B * WIDTH, "kv_len": 4 * B, "new_off": 4 * (B + 1), "left": 4,
        "parents": 4 * ROWS, "table_out": 4 * ROWS * WIDTH, "kv_len_out": 4 * ROWS, "refs_out": 4 * PAGES,
        "live": 4}
CALLS = {
    "reserve": (("refs", "table", "kv_len", "new_off", "left", "workspace"),
                ("refs", "table", "left", "workspace")),
    "release": (("refs", "table", "kv_len"), ("refs", "table")),
    "fork": (("refs", "table", "kv_len", "parents", "table_out", "kv_len_out", "refs_out", "left",
              "workspace"), ("table_out", "kv_len_out", "refs_out", "left", "workspace")),
    "compact": (("refs", "table", "table_out", "refs_out", "live", "workspace"),
                ("table_out", "refs_out", "live", "workspace")),
}


def size(call, name):
    if name == "workspace":
        refs, table = torch.empty(PAGES, device="meta"), torch.empty(B, WIDTH, device="meta")
        return sp.sparsp_pages_workspace_bytes(refs, table, ROWS if call == "fork" else 0)
    if call == "compact" and name == "table_out":
        return SIZE["table"]
    return SIZE[name]


def status(call, at, buffers=()):
    """Of the call with these addresses."""
    packed = b"".join(_BUFFER.pack(*x) for x in buffers) or None
    lib = sp.load_library()
    p = _PAGES.pack(at["refs"], at["table"], at.get("kv_len", 0), PAGES, PAGE, WIDTH, B)
    ws = (at.get("workspace"), size(call, "workspace"), None)
    if call == "reserve":
        rc = lib.sparsp_pages_reserve(p, at["new_off"], at["left"], *ws)
    elif call == "release":
        rc = lib.sparsp_pages_release(p, 5, 2, None)
    elif call == "fork":
        rc = lib.sparsp_pages_fork(p, at["parents"], ROWS, packed, len(buffers), at["table_out"],
                                   at["kv_len_out"], at["refs_out"], at["left"], *ws)
    else:
        rc = lib.sparsp_pages_compact(p, packed, len(buffers), at["table_out"], at["refs_out"],
                                      at["live"], *ws)
    return sp.STATUS[rc], lib.sparsp_last_error().decode()


def pairs():
    for call, (names, written) in CALLS.items():
        for i, a in enumerate(names):
            for b in names[:i]:
                if a in written or b in written:
                    yield call, a, b


@pytest.mark.parametrize("call,a,b", list(pairs()))
def test_overlapping_arrays_are_refused(call, a, b):
    """From the same address on, and by their last and first 16 bytes (of arrays that have as many)."""
    names = CALLS[call][0]
    for x, y in ((a, b), (b, a)):
        for off in {0, max(size(call, y) - 16, 0) & -16}:
            at = {n: (i + 1) * AT for i, n in enumerate(names)}
            at[x] = at[y] + off
            got, message = status(call, at)
            assert got == "SPARSP_E_INVALID", (x, y, off, message)
            assert "overlap" in message or "inputs" in message


@pytest.mark.parametrize("call,name", [(c, n) for c in ("fork", "compact") for n in CALLS[c][0]
                                       if (c, n) != ("fork", "left")])
def test_arrays_in_the_contents_are_refused(call, name):
    """At the first and in the last page of the second buffer."""
    at = {n: (i + 1) * AT for i, n in enumerate(CALLS[call][0])}
    first, second = 64 * AT, 65 * AT
    for off in (0, 48 * PAGES - 16):
        at[name] = second + off
        got, message = status(call, at, ((first, 16), (second, 48)))
        assert got == "SPARSP_E_INVALID" and "buffer 1 overlap" in message
    # The first bytes of the buffer are the array's last.
    at[name] = second - max(size(call, name) - 16, 0) // 16 * 16
    got, message = status(call, at, ((first - AT, 16), (second, 48)))
    assert got == "SPARSP_E_INVALID" and "buffer 1 overlap" in message


def test_page_numbers_in_the_contents_are_refused():
    lib = sp.load_library()
    for src, dst in ((2 * AT + 64 * PAGES - 16, AT), (AT, 2 * AT)):
        rc = lib.sparsp_pages_copy(_BUFFER.pack(2 * AT, 64), 1, PAGES, src, dst, 5, None)
        assert sp.STATUS[rc] == "SPARSP_E_INVALID" and "overlap" in lib.sparsp_last_error().decode()
