"""Refusals of the paged-cache calls, on the CPU: the binding checks tensors before any pointer is passed
on, the C entries check numbers before any CUDA call."""
import ctypes
import struct

import pytest
import torch


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def test_descriptors_have_the_sizes_of_the_c_structures(gorio):
    import paper_2607_04415_b200.paged as p
    assert (p._TABLES.size, p._STORE.size, p._ATTENTION.size) == (128, 144, 224)


@pytest.mark.parametrize("what", ["lengths", "q", "key_pages"])
def test_tensors_off_the_gpu_are_refused(gorio, what):
    i = torch.zeros(2, dtype=torch.int32)
    pages = torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16)
    rows = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(gorio.GorioError) as e:
        if what == "lengths":
            gorio.page_tables(i, i, torch.zeros((2, 2), dtype=torch.int32), i, i[:1], 16, 0)
        elif what == "q":
            gorio.paged_attention(rows, pages, pages, torch.zeros((1, 2), dtype=torch.int32), i[:1], i, 1)
        else:
            gorio.cache_store(rows, rows, pages, pages, torch.zeros(1, dtype=torch.int64))
    assert e.value.status == 1 and what in str(e.value)


def test_binding_refuses_wrong_shapes_types_and_strides(gorio):
    import paper_2607_04415_b200.paged as p
    cpu = -1                                               # what a tensor off the GPU has for a device index
    good = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    p._page_pair(good, good, cpu)
    for bad in (good[0], good.float(), good.half(), good[:, :1], good.transpose(2, 3)):
        with pytest.raises(gorio.GorioError):
            p._page_pair(good, bad, cpu)
    with pytest.raises(gorio.GorioError):
        p._page_pair(good, good, 0)
    with pytest.raises(gorio.GorioError):
        p._page_pair(good[..., ::2], good[..., ::2], cpu)
    rows = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    p._rows_3d("q", rows[:, 1:3], cpu, torch.bfloat16)
    for bad in (rows[0], rows.float(), rows[..., ::2], None):
        with pytest.raises(gorio.GorioError):
            p._rows_3d("q", bad, cpu, torch.bfloat16)
    v = torch.zeros(6, dtype=torch.int32)
    p._vector("lengths", v, cpu, 6)
    for bad, n in ((v, 5), (v[::2], 3), (v.long(), 6), (v[None], 6), ([0] * 6, 6)):
        with pytest.raises(gorio.GorioError):
            p._vector("lengths", bad, cpu, n)
    t = torch.zeros((3, 8), dtype=torch.int32)
    p._tables_2d(t[:, :4], 3, cpu)
    for bad, n in ((t, 4), (t[:, ::2], 3), (t[:, :0], 3), (t.long(), 3), (t[0], 3)):
        with pytest.raises(gorio.GorioError):
            p._tables_2d(bad, n, cpu)


A = 1 << 20        # an address that is never read: every call below is refused first


def _refused(lib, entry, packing, good, changes):
    """`good` itself would launch: it is not called.  Each change of one field has to be refused."""
    for at, value in changes:
        fields = list(good)
        fields[at] = value
        assert entry(packing.pack(*fields), None) == 1, (at, value)
        assert lib.gorio_last_error(None)


def test_c_entries_refuse_bad_numbers(gorio):
    import paper_2607_04415_b200.paged as p
    lib = gorio.load_library()
    for e in (lib.gorio_page_tables, lib.gorio_cache_store, lib.gorio_paged_attention):
        assert e(None, None) == 1
    assert lib.gorio_attention_check(None, None) == 1
    #         12 pointers, row stride; requests, width, capacity, page size, tokens, reserved
    tables = [A] * 12 + [4, 2, 4, 8, 16, 5, 0]
    _refused(lib, lib.gorio_page_tables, p._TABLES, tables,
             [(i, 0) for i in range(12)] + [(12, 3), (13, (1 << 20) + 1), (14, 0), (16, 0), (16, 1 << 29), (17, 1 << 31)])
    #        5 pointers, strides; tokens, heads, dim, pages, page size, reserved
    store = [A] * 5 + [128, 64, 128, 64, 2048, 1024, 64, 2048, 1024, 64] + [5, 2, 64, 9, 16, 0]
    _refused(lib, lib.gorio_cache_store, p._STORE, store,
             [(i, 0) for i in range(5)] + [(i, A + 8) for i in range(4)] + [(i, 66) for i in range(5, 15)] + [(17, 0), (17, 60), (18, 1 << 28), (19, 0)])
    #            10 pointers (slopes may be missing), strides; then requests, tokens, heads, key heads, dim, pages,
    #            page size, width, type, causal, window, max_new, scale, softcap
    attention = [A] * 4 + [0] + [A] * 3 + [0, A] + [256, 64, 256, 64, 2048, 1024, 64, 2048, 1024, 64, 4] + [2, 5, 4, 2, 64, 9, 16, 4, 0, 1, 0, 5, 0.1, 0.0]
    inf = float("inf")
    _refused(lib, lib.gorio_paged_attention, p._ATTENTION, attention,
             [(i, 0) for i in (0, 1, 2, 3, 5, 6, 7, 9)] + [(i, A + 8) for i in (0, 1, 2, 3, 9)] + [(i, 68) for i in range(10, 20)] +
             [(21, (1 << 20) + 1), (22, 1 << 31), (23, 0), (23, 5), (24, 0), (25, 80), (25, 256), (26, 1 << 28), (27, 0), (27, 12), (28, 0), (28, 1 << 27),
              (29, 2), (33, 0.0), (33, -1.0), (33, inf), (33, float("nan")), (34, -1.0), (34, inf)])


def test_nothing_to_do_is_no_error(gorio):
    import paper_2607_04415_b200.paged as p
    lib = gorio.load_library()
    assert lib.gorio_cache_store(p._STORE.pack(*([0] * 21)), None) == 0
    assert lib.gorio_paged_attention(p._ATTENTION.pack(*([0] * 33), 0.1, 0.0), None) == 0
    assert lib.gorio_attention_workspace_bytes(-1) == 0
    assert isinstance(p._TABLES, struct.Struct) and ctypes.sizeof(ctypes.c_void_p) == 8
