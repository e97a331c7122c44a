"""Scales of 8-bit rows that lie in one place: one scale for all rows where they are read, refused where every row writes its own."""
import ctypes as C

import pytest

import paper_2504_17307_amd as pkg
from test_rows_abi import B, EINVAL, OK, q8, rows


@pytest.mark.parametrize("n,stride,code", [(2, 0, EINVAL), (1000, 0, EINVAL), (0, 0, OK)])
def test_a_norm_does_not_write_its_rows_scales_to_one_place(n, stride, code):
    eps = C.byref(pkg.uccl_norm_opts(1e-6))
    assert pkg.load().uccl_norm_rows(q8(n, 16, scale_stride=stride), None, None, rows(n, 16), None, B, eps, None) == code


def test_the_binding_passes_the_refusal_on():
    import torch
    y, x = torch.zeros(3, 16, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(3, 16, dtype=torch.bfloat16)
    with pytest.raises(pkg.UcclError) as e:
        pkg.uccl_norm_rows(y, x, x[0], 1e-6, scales=torch.zeros(1, 1).expand(3, 1), stream=0)
    assert e.value.code == EINVAL


@pytest.mark.gpu
def test_one_scale_for_all_rows_is_read(gpu_lib):
    import torch
    from test_gpu_rows import aligned, gen, offsets_of, quantised
    g, counts, k, n = gen(6), [5, 0, 300], 200, 72
    (x, xs), (w, ws) = quantised(g, 305, k), quantised(g, 3 * n, k)
    off, got = offsets_of(counts), []
    for one_x, one_w in ((xs[:1].expand(305, 1), ws[:1].expand(3 * n, 1)), (xs[:1].repeat(305, 1), ws[:1].repeat(3 * n, 1))):
        y = aligned(305, n, torch.bfloat16)
        gpu_lib.uccl_group_product(y, x, w.unflatten(0, (3, n)), off, x_scales=one_x, w_scales=one_w)
        got.append(y)
    assert torch.equal(*got) and not bool(got[0].isnan().any())
