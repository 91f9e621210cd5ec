"""Refusals of the calls on shared prefixes and quantised caches, on the CPU: tensors in the binding, numbers in the C entries, before any CUDA
call."""
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
    import paper_2607_04415_b200.prefix as x
    import paper_2607_04415_b200.quantized as q
    assert (p._ATTENTION.size + x._PREFIX.size, q._ROWS.size, p._ATTENTION.size + q._SCALES.size) == (272, 216, 296)


def test_tensors_off_the_gpu_are_refused(gorio):
    i = torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    pages = torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16)
    codes, scales = pages.to(torch.float8_e4m3fn), torch.zeros((2, 1, 16))
    slots = torch.zeros(1, dtype=torch.int64)
    table = torch.zeros((1, 2), dtype=torch.int32)
    for call in (lambda: gorio.prefix_attention(rows, pages, pages, table, i[:1], i, table, i[:1], i, 1),
                 lambda: gorio.paged_attention_quantized(rows, codes, codes, scales, scales, table, i[:1], i, 1),
                 lambda: gorio.cache_store_quantized(rows, rows, codes, codes, scales, scales, slots),
                 lambda: gorio.cache_load_quantized(codes, codes, scales, scales, slots)):
        with pytest.raises(gorio.GorioError) as e:
            call()
        assert e.value.status == 1 and "CUDA" in str(e.value)


def test_binding_refuses_wrong_pages_and_scales(gorio):
    import paper_2607_04415_b200.quantized as q
    cpu = -1                                               # what a tensor off the GPU has for a device index
    codes, scales = torch.zeros((4, 2, 16, 64), dtype=torch.int8), torch.zeros((4, 2, 16))
    q._coded_pages(codes, codes, scales, scales, cpu)
    q._coded_pages(codes.transpose(1, 2).contiguous().transpose(1, 2), codes, scales, scales, cpu)
    for bad in (codes[0], codes.float(), codes.view(torch.float8_e4m3fn), codes[:, :1], codes.transpose(2, 3), codes[..., ::2], None):
        with pytest.raises(gorio.GorioError):
            q._coded_pages(codes, bad, scales, scales, cpu)
    for bad in (scales.half(), scales[:, :1], scales[..., None], None):
        with pytest.raises(gorio.GorioError):
            q._coded_pages(codes, codes, scales, bad, cpu)
    with pytest.raises(gorio.GorioError):
        q._coded_pages(codes, codes, scales, scales, 0)


A = 1 << 20        # an address that is never read: every call below is refused first


def _refused(lib, entry, packing, good, changes):
    """`good` itself would launch: it is not called.  Each change of one field has to be refused."""
    for at, value in changes:
        fields = list(good)
        fields[at] = value
        assert entry(packing(fields), None) == 1, (at, value)
        assert lib.gorio_last_error(None)


ATTENTION = [A] * 4 + [0] + [A] * 3 + [0, A] + [256, 64, 256, 64, 2048, 1024, 64, 2048, 1024, 64, 4] + [2, 5, 4, 2, 64, 9, 16, 4, 0, 1, 0, 5, 0.1, 0.0]
BAD_ATTENTION = ([(i, 0) for i in (0, 1, 2, 3, 5, 6, 7, 9)] + [(i, A + 8) for i in (0, 1, 2, 3, 9)] + [(i, 68) for i in range(10, 20)] +
                 [(21, (1 << 20) + 1), (22, 1 << 31), (23, 0), (23, 5), (24, 0), (25, 80), (25, 256), (26, 1 << 28), (27, 0), (27, 12), (28, 0), (28, 1 << 27),
                  (29, 2), (33, 0.0), (33, -1.0), (33, float("inf")), (33, float("nan")), (34, -1.0), (34, float("inf"))])


def test_c_entries_refuse_bad_numbers(gorio):
    import paper_2607_04415_b200.paged as p
    import paper_2607_04415_b200.prefix as x
    import paper_2607_04415_b200.quantized as q
    lib = gorio.load_library()
    for e in (lib.gorio_prefix_attention, lib.gorio_paged_attention_quantized, lib.gorio_cache_store_quantized, lib.gorio_cache_load_quantized):
        assert e(None, None) == 1
    n = len(ATTENTION)

    def both(more):
        return lambda f: p._ATTENTION.pack(*f[:n]) + more.pack(*f[n:])
    #         4 pointers, row stride; groups, width
    prefix = ATTENTION + [A] * 4 + [3, 2, 3]
    _refused(lib, lib.gorio_prefix_attention, both(x._PREFIX), prefix,
             BAD_ATTENTION + [(n + i, 0) for i in range(4)] + [(n + 3, A + 8), (n + 5, 0), (n + 5, (1 << 20) + 1), (n + 6, 0), (n + 6, 1 << 27), (n + 6, (1 << 27) - 3)])
    #        2 pointers, strides; format, reserved
    coded = ATTENTION + [A] * 2 + [32, 16, 1, 32, 16, 1, 0, 0]
    _refused(lib, lib.gorio_paged_attention_quantized, both(q._SCALES), coded,
             BAD_ATTENTION + [(i, 2056) for i in range(14, 20)] + [(n, 0), (n + 1, 0), (n, A + 2), (n + 1, A + 2), (n + 8, 2)])
    #       7 pointers, strides; tokens, heads, dim, pages, page size, type, format, reserved
    rows = [A] * 7 + [128, 64, 128, 64, 2048, 1024, 64, 2048, 1024, 64, 32, 16, 1, 32, 16, 1] + [5, 2, 64, 9, 16, 0, 0, 0]
    for entry in (lib.gorio_cache_store_quantized, lib.gorio_cache_load_quantized):
        _refused(lib, entry, lambda f: q._ROWS.pack(*f), rows,
                 [(i, 0) for i in range(7)] + [(i, A + 8) for i in range(4)] + [(4, A + 2), (5, A + 1)] + [(i, 68) for i in range(7, 11)] + [(i, 72) for i in range(11, 17)] +
                 [(23, 1 << 31), (24, 65537), (24, 1 << 31), (25, 0), (25, 72), (25, 272), (26, 1 << 28), (27, 0), (28, 2), (29, 2)])


def test_nothing_to_do_is_no_error(gorio):
    import paper_2607_04415_b200.paged as p
    import paper_2607_04415_b200.prefix as x
    import paper_2607_04415_b200.quantized as q
    lib = gorio.load_library()
    none = p._ATTENTION.pack(*([0] * 33), 0.1, 0.0)
    assert lib.gorio_prefix_attention(none + x._PREFIX.pack(*([0] * 7)), None) == 0
    assert lib.gorio_paged_attention_quantized(none + q._SCALES.pack(*([0] * 10)), None) == 0
    assert lib.gorio_cache_store_quantized(q._ROWS.pack(*([0] * 31)), None) == 0
    assert lib.gorio_cache_load_quantized(q._ROWS.pack(*([0] * 31)), None) == 0
    assert lib.gorio_prefix_scratch_bytes(-1, 5, 4, 64) == 0
