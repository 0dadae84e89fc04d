"""hs_kv_append of keys and values whose strides differ where they mean
nothing: along an axis of length 1."""
import pytest
import torch

import kv_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H", [(1, 3), (5, 1), (1, 1)])
@pytest.mark.parametrize("swap", [False, True])
def test_axes_of_length_one(T, H, swap):
    d = 64
    wide = torch.randn((T, H, 5 * d), device="cuda").to(torch.bfloat16)
    x = torch.randn((T, H, d), device="cuda").to(torch.bfloat16)
    # the same strides along axes of more than one, any along the others
    by = [H * d if T > 1 else 7 * d + 3, d if H > 1 else 3 * d + 1, 1]
    y = torch.empty(T * H * d + 16, dtype=torch.bfloat16, device="cuda").as_strided((T, H, d), by)
    y.copy_(wide[..., :d])
    k, v = (y, x) if swap else (x, y)
    got, want = (hs.KvCache(2, 16, H, d) for _ in range(2))
    slots = torch.arange(3, 3 + T, dtype=torch.int32, device="cuda")
    for c in (got, want):
        c.k.view(torch.uint8).zero_()
        c.v.view(torch.uint8).zero_()
    hs.hs_kv_append(got, k, v, slots)
    hs.hs_kv_append(want, k.clone(memory_format=torch.contiguous_format),
                    v.clone(memory_format=torch.contiguous_format), slots)
    hs.hs_get_device_error()
    for a, b in ((got.k, want.k), (got.v, want.v)):
        assert (ref.to_bytes(a) == ref.to_bytes(b)).all()
    assert torch.equal(got.k_scale[0], want.k_scale[0]) and torch.equal(got.v_scale[0], want.v_scale[0])
    assert (ref.to_bytes(got.v)[0, :, 3:3 + T] != 0).any()


def test_strides_that_matter_still_have_to_be_the_same():
    c = hs.KvCache(2, 16, 2, 64)
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda")[..., :64]
    with pytest.raises(ValueError):
        hs.hs_kv_append(c, x, wide, torch.arange(3, dtype=torch.int32, device="cuda"))
