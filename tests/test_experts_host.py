"""Host-side checks of the entry points for layers of experts and clipped gradients, without a GPU: sizes of descriptors and workspaces, and
refusals before anything is launched."""
import ctypes

import pytest
import torch

from paper_1811_12019_amd import binding as kb

INVALID, WORKSPACE, TOO_LARGE = kb.KFAC_ERR_INVALID_ARG, kb.KFAC_ERR_WORKSPACE, kb.KFAC_ERR_TOO_LARGE
P = ctypes.c_void_p
A, B, C, D = P(0x1000000), P(0x2000000), P(0x3000000), P(0x4000000)     # never dereferenced: every call below fails before a launch


def desc(tokens=8, choices=2, experts=4, dim=64, dtype=kb.KFAC_BF16, ld_token=0, ld_row=0, ld_grad=0):
    return kb.kfac_expert_desc(tokens, choices, experts, dim, dtype, ld_token, ld_row, ld_grad)


def fdesc(rows=64, experts=4, dim=64, dtype=kb.KFAC_BF16, has_bias=0, packed=0, ld=0):
    return kb.kfac_expert_factor_desc(rows, experts, dim, dtype, has_bias, packed, ld)


def test_struct_sizes_match_header():
    assert ctypes.sizeof(kb.kfac_grad_item) == 8 + 8 + 8 + 8
    assert ctypes.sizeof(kb.kfac_expert_desc) == 24 + 3 * 8
    assert ctypes.sizeof(kb.kfac_expert_factor_desc) == 6 * 4 + 8


BAD_ROUTES = [dict(tokens=-1), dict(choices=0), dict(choices=65), dict(experts=0), dict(experts=1025), dict(tokens=1 << 30, choices=2)]
BAD_ROWS = BAD_ROUTES + [dict(dim=0), dict(dim=(1 << 20) + 1), dict(dtype=3), dict(ld_token=63), dict(ld_row=63), dict(ld_row=-1),
                         dict(ld_token=(1 << 28) + 1), dict(ld_grad=63), dict(ld_grad=(1 << 28) + 1)]


@pytest.mark.parametrize("change", BAD_ROUTES, ids=str)
def test_sort_refuses(change):
    lib = kb.load_library()
    d = desc(**change)
    assert lib.kfac_expert_sort_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.kfac_expert_sort(ctypes.byref(d), A, B, C, D, None, 0, None) == INVALID


def test_sort_refuses_pointers():
    lib = kb.load_library()
    d = ctypes.byref(desc())
    assert lib.kfac_expert_sort(None, A, B, C, D, None, 0, None) == INVALID
    assert lib.kfac_expert_sort(d, None, B, C, D, None, 0, None) == INVALID
    assert lib.kfac_expert_sort(d, A, None, C, D, None, 0, None) == INVALID
    assert lib.kfac_expert_sort(d, A, B, C, None, None, 0, None) == INVALID
    assert lib.kfac_expert_sort(d, P(0x1000002), B, C, D, None, 0, None) == INVALID
    assert lib.kfac_expert_sort(d, A, B, C, A, None, 0, None) == INVALID                 # in place
    assert lib.kfac_expert_sort(d, A, B, P(0x4000020), D, None, 0, None) == INVALID      # order inside place
    big = ctypes.byref(desc(tokens=100000))
    need = lib.kfac_expert_sort_workspace_bytes(big)
    assert need > 0 and need % 256 == 0
    assert lib.kfac_expert_sort(big, A, B, C, D, None, 0, None) == WORKSPACE
    assert lib.kfac_expert_sort(big, A, B, C, D, P(0x5000010), 1 << 30, None) == WORKSPACE
    assert lib.kfac_expert_sort(big, A, B, C, D, P(0x5000000), need - 1, None) == WORKSPACE


@pytest.mark.parametrize("change", BAD_ROWS, ids=str)
def test_rows_refuse(change):
    lib = kb.load_library()
    d = ctypes.byref(desc(**change))
    assert lib.kfac_expert_dispatch(d, A, B, C, None) == INVALID
    assert lib.kfac_expert_combine(d, A, None, B, C, None) == INVALID
    assert lib.kfac_expert_combine_backward(d, A, B, None, C, D, None, None) == INVALID


def test_rows_refuse_pointers():
    lib = kb.load_library()
    d = ctypes.byref(desc())
    assert lib.kfac_expert_dispatch(None, A, B, C, None) == INVALID
    for bad in (None, P(0x1000001)):
        assert lib.kfac_expert_dispatch(d, bad, B, C, None) == INVALID
        assert lib.kfac_expert_dispatch(d, A, bad, C, None) == INVALID
        assert lib.kfac_expert_dispatch(d, A, B, bad, None) == INVALID
        assert lib.kfac_expert_combine(d, bad, None, B, C, None) == INVALID
        assert lib.kfac_expert_combine(d, A, None, bad, C, None) == INVALID
        assert lib.kfac_expert_combine(d, A, None, B, bad, None) == INVALID
        assert lib.kfac_expert_combine_backward(d, bad, B, None, C, D, None, None) == INVALID
        assert lib.kfac_expert_combine_backward(d, A, bad, None, C, D, A, None) == INVALID       # dweights without ys
        assert lib.kfac_expert_combine_backward(d, A, B, None, bad, D, None, None) == INVALID
        assert lib.kfac_expert_combine_backward(d, A, B, None, C, bad, None, None) == INVALID
    assert lib.kfac_expert_combine(d, A, P(0x2000002), B, C, None) == INVALID
    assert lib.kfac_expert_dispatch(d, A, B, A, None) == INVALID                          # in place
    assert lib.kfac_expert_dispatch(d, A, B, P(0x1000000 + 8 * 128 - 2), None) == INVALID  # the last token's last element
    assert lib.kfac_expert_combine(d, A, None, B, A, None) == INVALID
    assert lib.kfac_expert_combine_backward(d, A, B, None, C, A, None, None) == INVALID
    assert lib.kfac_expert_combine_backward(d, A, B, None, C, B, D, None) == INVALID       # ys and dys
    many = ctypes.byref(desc(tokens=1 << 20, choices=1, dim=1 << 20))
    assert lib.kfac_expert_dispatch(many, A, B, C, None) == TOO_LARGE
    for tokens, dim in [(1 << 29, 8), (200000000, 80)]:                                   # more threads than a launch has, of short rows
        far = [P(k << 44) for k in range(1, 5)]
        assert lib.kfac_expert_combine_backward(ctypes.byref(desc(tokens=tokens, choices=1, dim=dim)), far[0], far[1], None, far[2], far[3], None, None) == TOO_LARGE


def test_nothing_to_do_launches_nothing():
    lib = kb.load_library()
    none = ctypes.byref(desc(tokens=0))
    assert lib.kfac_expert_dispatch(none, None, None, None, None) == kb.KFAC_OK
    assert lib.kfac_expert_combine(none, None, None, None, None, None) == kb.KFAC_OK
    assert lib.kfac_expert_combine_backward(none, None, None, None, None, None, None, None) == kb.KFAC_OK


@pytest.mark.parametrize("change", [dict(rows=-1), dict(experts=0), dict(experts=1025), dict(dim=0), dict(dim=32767), dict(dtype=-1),
                                    dict(has_bias=2), dict(packed=2), dict(ld=63), dict(ld=-64), dict(ld=(1 << 28) + 8)], ids=str)
def test_factor_refuses(change):
    lib = kb.load_library()
    d = ctypes.byref(fdesc(**change))
    assert lib.kfac_expert_factor_workspace_bytes(d) == 0
    assert lib.kfac_expert_factor(d, A, B, 0.0, C, None, 0.0, None, 0, None) == INVALID


def test_factor_refuses_pointers():
    lib = kb.load_library()
    call = lib.kfac_expert_factor
    d = ctypes.byref(fdesc())
    assert lib.kfac_expert_factor_workspace_bytes(d) == 0                                # whole vectors, too few rows for two ranges
    assert call(None, A, B, 0.0, C, None, 0.0, None, 0, None) == INVALID
    assert call(d, None, B, 0.0, C, None, 0.0, None, 0, None) == INVALID
    assert call(d, P(0x1000008), B, 0.0, C, None, 0.0, None, 0, None) == INVALID         # whole vectors, off the 16-byte grid
    assert call(d, A, None, 0.0, C, None, 0.0, None, 0, None) == INVALID
    assert call(d, A, B, 0.0, None, None, 0.0, None, 0, None) == INVALID
    assert call(d, A, B, 0.0, C, D, 0.5, None, 0, None) == INVALID                       # both destinations
    assert call(d, A, B, 0.0, None, D, 1.5, None, 0, None) == INVALID
    assert call(d, A, B, 0.0, None, D, float("nan"), None, 0, None) == INVALID
    assert call(ctypes.byref(fdesc(packed=1)), A, B, 0.0, None, D, 0.5, None, 0, None) == INVALID
    odd = ctypes.byref(fdesc(dim=63))                                                    # copied first
    need = lib.kfac_expert_factor_workspace_bytes(odd)
    assert need == 64 * 64 * 2
    assert call(odd, A, B, 0.0, C, None, 0.0, None, 0, None) == WORKSPACE
    assert call(odd, A, B, 0.0, C, None, 0.0, P(0x5000080), 1 << 30, None) == WORKSPACE
    many = ctypes.byref(fdesc(rows=100000))                                              # several ranges
    assert lib.kfac_expert_factor_workspace_bytes(many) > 0
    assert call(many, A, B, 0.0, C, None, 0.0, None, 0, None) == WORKSPACE
    huge = fdesc(rows=1 << 20, experts=1024, dim=32760)
    assert call(ctypes.byref(huge), A, B, 0.0, C, None, 0.0, P(0x5000000), 1 << 62, None) == TOO_LARGE


def items(*rows):
    return (kb.kfac_grad_item * len(rows))(*[kb.kfac_grad_item(*r) for r in rows])


def test_norm_and_clip_refuse():
    lib = kb.load_library()
    norm, clip = lib.kfac_grad_norm_batched, lib.kfac_grad_clip_batched
    ok = items((0x1000000, 0x2000000, 5000, kb.KFAC_F32), (0x3000000, None, 7, kb.KFAC_BF16), (None, None, 0, kb.KFAC_F16))
    need = lib.kfac_grad_norm_workspace_bytes(ok, 3)
    assert need == 256                                                                   # 2 + 1 chunks, a double each
    assert norm(ok, 3, None, A, need, None) == INVALID
    assert norm(ok, 3, A, None, 0, None) == WORKSPACE
    assert norm(ok, 3, A, P(0x5000010), 1 << 20, None) == WORKSPACE
    assert norm(ok, 3, A, B, need - 1, None) == WORKSPACE
    assert norm(None, 1, A, B, need, None) == INVALID
    assert norm(ok, -1, A, B, need, None) == INVALID
    assert clip(ok, 3, -1.0, None, A, B, need, None) == INVALID
    assert clip(ok, 3, float("nan"), None, A, B, need, None) == INVALID
    assert clip(ok, 3, 1.0, None, None, B, need, None) == INVALID                        # nowhere for the norm
    assert clip(ok, 3, 1.0, A, B, None, 0, None) == INVALID                              # both a given norm and a place for it
    assert clip(ok, 3, 1.0, None, A, None, 0, None) == WORKSPACE
    for bad in ((None, None, 5, kb.KFAC_F32), (0x1000002, None, 5, kb.KFAC_F32), (0x1000001, None, 5, kb.KFAC_BF16),
                (0x1000000, None, -1, kb.KFAC_F32), (0x1000000, None, 5, 7)):
        assert norm(items(bad), 1, A, B, 256, None) == INVALID, bad
        assert clip(items(bad), 1, 1.0, None, A, B, 256, None) == INVALID, bad
    for out in (0x1000010, 0x1000000 - 16, 0x2000002):                                   # overlapping, or off its elements' grid
        bad = items((0x1000000, out, 5000, kb.KFAC_F32))
        assert clip(bad, 1, 1.0, None, A, B, 256, None) == INVALID, out
    assert norm(items((0x1000000, None, 1 << 43, kb.KFAC_BF16)), 1, A, B, 256, None) == TOO_LARGE
    assert lib.kfac_grad_norm_workspace_bytes(items((0x1000000, None, 1 << 43, kb.KFAC_BF16)), 1) == 0
    assert clip(items((None, None, 0, kb.KFAC_F32)), 1, 1.0, A, None, None, 0, None) == kb.KFAC_OK      # nothing to do, no launch
    assert clip(None, 0, 1.0, A, None, None, 0, None) == kb.KFAC_OK


def test_norm_scratch_does_not_grow_with_the_gradients():
    lib = kb.load_library()
    for count, n in ((1, 1 << 20), (1, 1 << 40), (300, 1 << 22), (1000, 1 << 30), (2000, 3)):
        need = lib.kfac_grad_norm_workspace_bytes(items(*[(0x1000000, None, n, kb.KFAC_F32)] * count), count)
        assert 256 <= need <= 8 * (1024 + count) + 256


def test_binding_refuses_host_memory():
    cpu = torch.zeros(4)
    with pytest.raises(kb.KfacError) as e:
        kb.GradBatch([cpu], device="cpu")
    assert e.value.status == INVALID and "GPU" in str(e.value)
    with pytest.raises(kb.KfacError):
        kb.ExpertRoute(4, 2, 3, device="cpu")
    with pytest.raises(kb.KfacError):
        kb.ExpertFactors(4, 2, 3, torch.float32, device="cpu")


def test_rows_with_gaps_that_overlap_are_refused():
    """Written rows that share an element with rows that are read, whatever lies between the rows of either."""
    lib = kb.load_library()
    # 8 tokens, 16 rows of 64 bfloat16 (128 bytes); rows `ld` elements apart
    def dispatch(ld_token, ld_row, off):
        d = desc(ld_token=ld_token, ld_row=ld_row)
        return lib.kfac_expert_dispatch(ctypes.byref(d), A, C, P(0x1000000 + off), None)

    refused = [(128, 0, 0), (128, 0, 126), (128, 0, 7 * 256), (128, 0, 7 * 256 + 126), (128, 0, -2046),     # tokens with gaps, rows without
               (0, 128, 126), (0, 128, 2), (0, 128, -15 * 256), (0, 128, -15 * 256 - 126),                  # rows with gaps, tokens without
               (128, 128, 126), (128, 128, 256), (128, 128, 130), (128, 128, 7 * 256), (128, 128, 7 * 256 + 126), (128, 128, -126),   # both, as far apart
               (128, 128, -15 * 256 - 126), (128, 128, -3 * 256 + 2), (192, 192, 64), (192, 192, -384 - 100)]
    for ld_token, ld_row, off in refused:
        assert dispatch(ld_token, ld_row, off) == INVALID, (ld_token, ld_row, off)
    wide = ctypes.byref(desc(ld_token=128, ld_row=128, ld_grad=128))
    near = P(0x2000000 + 64)
    assert lib.kfac_expert_combine(wide, A, None, C, P(0x1000000 + 64), None) == INVALID
    assert lib.kfac_expert_combine_backward(wide, A, B, None, C, P(0x1000000 + 256 - 2), None, None) == INVALID
    assert lib.kfac_expert_combine_backward(wide, A, B, None, C, near, D, None) == INVALID
    one = ctypes.byref(desc(tokens=1, choices=1, ld_token=128, ld_row=4096))                                # one row each: gaps are of no matter
    assert lib.kfac_expert_dispatch(one, A, C, P(0x1000000 + 126), None) == INVALID
