"""wk_page_store: copies are exact, rows in 8 bits are the nearest codes under the least power of two, and nothing else is touched."""
import math

import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


def bits(x):
    return x.contiguous().view(torch.uint8)


def rows(n, heads, d, dtype, seed, wide=False):
    """K and V rows, contiguous or as slices of wider rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if not wide:
        return [torch.randn((n, heads, d), generator=g, device="cuda").to(dtype) for _ in range(2)]
    both = torch.randn((n, 3 * heads, d), generator=g, device="cuda").to(dtype)
    return [both[:, heads:2 * heads], both[:, 2 * heads:]]


@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("n,heads,d,page,layout,wide", [
    (1, 1, 64, 1, "tokens", False), (1, 12, 128, 16, "tokens", True), (37, 5, 64, 7, "heads", True), (100, 8, 128, 16, "paired", False),
    (1000, 1, 128, 24, "heads", False), (515, 40, 128, 16, "tokens", False), (33, 130, 64, 16, "tokens", True),
])
def test_rows_reach_their_slots(kv, type_, n, heads, d, page, layout, wide):
    from paper_2605_22718_b200 import PagedKV
    n_pages = -(-n // page) + 2
    K, V, ke, ve = lib.cache(type_, n_pages, page, heads, d, seed=1, layout=layout)
    before = [x.clone() for x in (K, V)] + [x.clone() if x is not None else None for x in (ke, ve)]
    src = lib.TYPES[type_] if type_ != "e4m3" else torch.float16 if n % 2 else torch.bfloat16
    new = rows(n, heads, d, src, 2, wide)
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(3))[:n].int().cuda()
    slots[n // 2] = -1 if n > 1 else slots[0]
    PagedKV(kv, K, V, ke, ve).page_store(new[0], new[1], slots)
    assert kv.poll_status() == (0, 0)
    put = slots >= 0
    at = (slots[put] // page).long(), (slots[put] % page).long()
    for x, e, old, old_e, r in ((K, ke, before[0], before[2], new[0]), (V, ve, before[1], before[3], new[1])):
        if type_ == "e4m3":
            value, byte = lib.quantise(r[put])
            assert torch.equal(x[at].double().cpu(), value)
            assert torch.equal(e.transpose(1, 2)[at].cpu(), byte)
            old_e.transpose(1, 2)[at] = byte.cuda()
            assert torch.equal(e, old_e)
            old[at] = value.float().to(torch.float8_e4m3fn).cuda()
        else:
            old[at] = r[put]
        assert torch.equal(bits(x), bits(old))      # the rows, and every other byte as it was


@pytest.mark.parametrize("src", [torch.bfloat16, torch.float16])
def test_rows_in_8_bits_where_rounding_decides(kv, src):
    """Largest magnitudes on either side of 448 * 2^e, ties between codes, codes below the normal numbers, zeros, the type's extremes."""
    from paper_2605_22718_b200 import PagedKV
    big = torch.finfo(src).max
    tiny = torch.finfo(src).smallest_normal
    x = torch.zeros((12, 1, 128), dtype=torch.float64)
    ladder = torch.arange(128, dtype=torch.float64)
    x[0, 0] = ladder / 128 * 1.75                                   # amax just below 1.75 * 2^0
    x[1, 0] = ladder / 127 * 1.75                                   # exactly 1.75
    x[2, 0] = ladder / 127 * 1.7578125                              # the next bf16 above it
    x[3, 0] = (ladder - 64) * 17 / 16                               # ties of many binades
    x[4, 0, 5] = -448.0
    x[4, 0, 6:40] = torch.pow(2.0, -torch.arange(34, dtype=torch.float64))      # down to below the codes
    x[4, 0, 40:74] = 1.5 * torch.pow(2.0, -torch.arange(34, dtype=torch.float64))
    x[5, 0, 3] = big
    x[5, 0, 4] = -big / 3
    x[6, 0, 7] = tiny
    x[6, 0, 8] = tiny / 4
    x[7, 0] = tiny / 8 * (ladder % 7)
    x[9, 0] = -0.0
    x[10, 0] = torch.where(ladder % 2 == 0, 1.0, -1.0) * torch.pow(2.0, -(ladder % 24))
    x[11, 0] = 1.0
    r = x.to(src).cuda()
    K, V, ke, ve = lib.cache("e4m3", 2, 8, 1, 128)
    PagedKV(kv, K, V, ke, ve).page_store(r, -r, torch.arange(12, dtype=torch.int32, device="cuda"))
    value, byte = lib.quantise(r)
    got, got_e = K.view(16, 1, 128)[:12].double().cpu(), ke.transpose(1, 2).reshape(16, 1)[:12].cpu()
    assert torch.equal(got, value) and torch.equal(got_e, byte)
    assert torch.equal(V.view(16, 1, 128)[:12].double().cpu(), -value)
    assert byte[8].item() == byte[9].item() == 127 and kv.poll_status() == (0, 0)


def test_values_that_are_not_finite(kv):
    from paper_2605_22718_b200 import PagedKV, WK_DEV_NONFINITE
    r, = rows(3, 2, 64, torch.bfloat16, 5)[:1]
    r[0, 0, 9], r[1, 1, 0], r[1, 1, 63], r[2, 0] = math.inf, math.nan, -math.inf, math.inf
    K, V, ke, ve = lib.cache("e4m3", 1, 4, 2, 64)
    PagedKV(kv, K, V, ke, ve).page_store(r, r, torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda"))
    value, byte = lib.quantise(r)
    torch.testing.assert_close(K[0, [2, 0, 1]].double().cpu(), value, rtol=0, atol=0, equal_nan=True)
    assert torch.equal(ke[0].t()[[2, 0, 1]].cpu(), byte)
    assert kv.poll_status()[1] == WK_DEV_NONFINITE
    B, BV, _, _ = lib.cache("bf16", 1, 4, 2, 64)                    # as they are in a cache of 16 bits
    PagedKV(kv, B, BV).page_store(r, r, torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(bits(B[0, [2, 0, 1]]), bits(r)) and kv.poll_status() == (0, 0)


@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
def test_slots_out_of_range_are_skipped(kv, type_):
    from paper_2605_22718_b200 import PagedKV, WK_DEV_BAD_SLOT
    K, V, ke, ve = lib.cache(type_, 3, 8, 2, 128)
    old = [K.clone(), V.clone()]
    new = rows(6, 2, 128, torch.bfloat16, 7)
    c = PagedKV(kv, K, V, ke, ve)
    c.page_store(*new, torch.full((6,), -1, dtype=torch.int32, device="cuda"))
    assert kv.poll_status() == (0, 0)
    c.page_store(*new, torch.tensor([24, -2, 2 ** 31 - 1, -2 ** 31, 25, -1], dtype=torch.int32, device="cuda"))
    assert kv.poll_status()[1] == WK_DEV_BAD_SLOT
    assert torch.equal(bits(K), bits(old[0])) and torch.equal(bits(V), bits(old[1]))


def test_a_cache_past_32_bits(kv):
    """Pages beyond 4 GB (and 2^31 elements) of a cache."""
    from paper_2605_22718_b200 import PagedKV
    n_pages, page = 40000, 64
    K = torch.empty((n_pages, page, 8, 128), dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    assert K.numel() > 2 ** 31
    new = rows(3, 8, 128, torch.bfloat16, 9)
    slots = torch.tensor([n_pages * page - 1, 3 * 2 ** 19, 2 ** 21 + 5], dtype=torch.int32, device="cuda")
    for x in (K, V):
        x.view(-1, 8, 128)[slots.long()] = 0
    PagedKV(kv, K, V).page_store(*new, slots)
    assert torch.equal(K.view(-1, 8, 128)[slots.long()], new[0]) and torch.equal(V.view(-1, 8, 128)[slots.long()], new[1])
    assert kv.poll_status() == (0, 0)
