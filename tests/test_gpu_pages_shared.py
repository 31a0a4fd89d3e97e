"""What the page calls promise of memory, of old contents and of shortages, against loops over lists."""

import pytest
import torch

import paper_2609_32197_amd as sp
from tests.test_gpu_pages import Pool, ints

pytestmark = pytest.mark.gpu
I32 = torch.int32


def test_arrays_side_by_side(gpu):
    """Every array of a turn and a compaction in one tensor, one right behind the other."""
    pages, width, kv, parents = 60, 9, (100, 37, 144, 16), [2, 2, 0, -1, 1]
    p = Pool(11, pages, 16, width, kv)
    rows = len(parents)
    sizes = dict(refs=(pages,), table=(4, width), kv=(4,), parents=(rows,), off=(rows + 1,),
                 table_out=(rows, width), kv_out=(rows,), refs_out=(pages,), left=(1,),
                 table_end=(rows, width), refs_end=(pages,), live=(1,))
    total = sum(torch.Size(s).numel() for s in sizes.values())
    ws = sp.sparsp_pages_workspace_bytes(ints(p.refs), ints(p.table), rows)
    room = torch.full((total + (-total) % 4 + ws // 4 + 1,), -77, dtype=I32, device="cuda")
    at, x = 0, {}
    for name, shape in sizes.items():
        n = torch.Size(shape).numel()
        x[name] = room[at:at + n].view(shape)
        at += n
    work = room[at + (-at) % 4:][:-(-ws // 4)]
    for name, value in (("refs", p.refs), ("table", p.table), ("kv", p.kv), ("parents", parents),
                        ("off", [0, 3, 6, 6, 8, 9])):
        x[name].copy_(ints(value))
    sp.sparsp_pages_fork(x["refs"], x["table"], x["kv"], x["parents"], 16, page_table_out=x["table_out"],
                         kv_len_out=x["kv_out"], refs_out=x["refs_out"], left=x["left"], workspace=work)
    t, k, r, left, _ = p.fork(parents)
    assert x["refs"].tolist() == p.refs and x["table"].tolist() == p.table and x["kv"].tolist() == p.kv
    assert x["table_out"].tolist() == t and x["kv_out"].tolist() == k
    assert x["refs_out"].tolist() == r and int(x["left"]) == left
    p.table, p.kv, p.refs = t, k, r
    sp.sparsp_pages_release(x["refs_out"], x["table_out"], x["kv_out"], 16, window=40, sinks=3)
    p.release(p.kv, 40, 3)
    new = [3, 3, 0, 2, 1]
    p.kv = [min(a + b, 16 * width) for a, b in zip(p.kv, new)]
    x["kv_out"].copy_(ints(p.kv))
    sp.sparsp_pages_reserve(x["refs_out"], x["table_out"], x["off"], x["kv_out"], 16, left=x["left"],
                            workspace=work)
    assert int(x["left"]) == p.reserve(new)
    assert x["table_out"].tolist() == p.table and x["refs_out"].tolist() == p.refs
    sp.sparsp_pages_compact(x["refs_out"], x["table_out"], page_table_out=x["table_end"],
                            refs_out=x["refs_end"], live=x["live"], workspace=work)
    t, r, n, _ = p.compact()
    assert x["table_end"].tolist() == t and x["refs_end"].tolist() == r and int(x["live"]) == n
    assert x["off"].tolist() == [0, 3, 6, 6, 8, 9] and x["parents"].tolist() == parents


def test_a_pool_of_no_pages_is_refused(gpu):
    none, table, kv = ints([]), ints([[0]]), ints([1])
    x = torch.zeros(0, 8, device="cuda")
    for call in (lambda: sp.sparsp_pages_fork(none, table, kv, ints([0]), 16, x),
                 lambda: sp.sparsp_pages_compact(none, table, x),
                 lambda: sp.sparsp_pages_copy(ints([0]), ints([0]), x)):
        with pytest.raises(sp.SparspError):
            call()
