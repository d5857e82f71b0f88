"""What the binding of paged caches asks of torch and says of its arguments."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2609_30738_amd import _lib

FOUR_BITS = "float4_e2m1fn_x2"


def test_8_bit_caches_do_without_4_bit_types(monkeypatch):
    """Where torch has no 4-bit type, an 8-bit cache's tensors are looked at as ever (here they are the host's, which is
    refused as such), and a 4-bit cache is refused."""
    monkeypatch.delattr(torch, FOUR_BITS)
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for dtype in (torch.float8_e4m3fn, torch.int8):
        pool = torch.zeros(8, 2, 16, 64, dtype=torch.uint8).view(dtype)
        with pytest.raises(ValueError, match="table must be a contiguous"):
            _lib.PagedCache("bf16", 4, pool, pool, torch.zeros(8, 2), torch.zeros(8, 2), table, lens)
    for qtype in ("e4m3", "int8"):
        with pytest.raises(ValueError, match="table must be a contiguous"):
            _lib.PagedCache.allocate("bf16", qtype, 4, 2, 64, 16, 8, 2, 4, device="cpu")
    with pytest.raises(ValueError, match=FOUR_BITS):
        _lib.PagedCache.allocate("bf16", "e2m1", 4, 2, 64, 16, 8, 2, 4, device="cpu")
    pool = torch.zeros(8, 2, 16, 32, dtype=torch.uint8)
    with pytest.raises(ValueError, match="k and v must be"):
        _lib.PagedCache("bf16", 4, pool, pool, pool, pool, table, lens)


def test_refusals_name_the_place():
    """A tensor on the host is refused as one that is not on a GPU, by no index that the caller never gave."""
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    pool = torch.zeros(8, 2, 16, 64, dtype=torch.int8)
    with pytest.raises(ValueError, match="^table must be a contiguous torch.int32 tensor of at least 0 elements on a GPU$"):
        _lib.PagedCache("bf16", 4, pool, pool, torch.zeros(8, 2), torch.zeros(8, 2), table, lens)
    for index, place in ((1, "cuda:1"), (-2, "a GPU")):
        with pytest.raises(ValueError, match=rf"^x must be a torch.float32 tensor \[tokens, 2, 64\] on {place}$"):
            _lib._token_rows(torch.zeros(3, 2, 64), torch.float32, index, 2, 64, "x")


@pytest.mark.gpu
@pytest.mark.parametrize("qtype", ["e4m3", "int8"])
def test_appending_without_4_bit_types(monkeypatch, qtype):
    monkeypatch.delattr(torch, FOUR_BITS)
    rng = np.random.default_rng(1)
    pc = _lib.PagedCache.allocate("bf16", qtype, 4, 2, 64, 16, 4, 1, 4)
    x = torch.from_numpy(rng.standard_normal((20, 2, 64)).astype(np.float32)).cuda().bfloat16()
    codes, scale = np.zeros((4, 2, 16, 64), np.uint8), np.zeros((4, 2))
    _lib.paged_append(pc, x, x.clone(), torch.arange(20, dtype=torch.int32, device="cuda"))
    paged.append(codes, scale, x.double().cpu().numpy(), np.arange(20), qtype)
    got = pc.k.view(torch.uint8).cpu().numpy()
    assert np.array_equal(got[0], codes[0]) and np.array_equal(got[1, :, :4], codes[1, :, :4])
    assert np.array_equal(pc.k_scale[:2].double().cpu().numpy(), scale[:2])
