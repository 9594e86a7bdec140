"""wk_paged_attention on rows that are not finite, in every type, and on weights too small for theirs to show."""
import math

import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[50, 50, 50], [5000, 70, 999]])
@pytest.mark.parametrize("place", [0, 17, 49])
def test_codes_that_are_not_numbers(kv, d, lens, place):
    """As page_store writes them: a key with one spoils its head's rows and no other, a value with one its column."""
    from paper_2605_22718_b200 import PagedKV, WK_DEV_NONFINITE
    page, heads = 16, 4
    n_pages = sum(-(-n // page) for n in lens)
    c = PagedKV.empty(kv, n_pages, page, heads, d, torch.float8_e4m3fn)
    tables = lib.tables_for(lens, page, n_pages, max(-(-n // page) for n in lens))
    g = torch.Generator(device="cuda").manual_seed(place)
    for r, n in enumerate(lens):
        t = torch.arange(n, device="cuda")
        K, V = (torch.randn((n, heads, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        if r == 0:
            K[place, 1, 5] = math.inf
            V[place, 2, 6], V[n - 1, 3, 7] = math.nan, -math.inf
        c.page_store(K, V, (tables[r].long()[t // page] * page + t % page).int())
    assert kv.poll_status()[1] == WK_DEV_NONFINITE
    Q = torch.randn((len(lens), 2 * heads, d), generator=g, device="cuda").to(torch.bfloat16)
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    lse = torch.empty(Q.shape[:2], device="cuda")
    O = c.paged_attention(Q, tables, dev, lse_out=lse)
    nan = torch.zeros(O.shape, dtype=torch.bool, device="cuda")
    nan[0, 2:4], nan[0, 4:6, 6], nan[0, 6:8, 7] = True, True, True
    assert torch.equal(O.isnan(), nan) and torch.equal(lse.isnan(), nan.all(-1))
    lib.assert_attends(O, lse, lib.attend(Q, c.K, c.V, c.K_exp, c.V_exp, tables, lens))
    assert kv.poll_status() == (0, 0)


@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
def test_queries_that_are_not_finite(kv, type_):
    """They spoil their own row."""
    from paper_2605_22718_b200 import PagedKV
    K, V, ke, ve = lib.cache(type_, 20, 16, 2, 128)
    tables = torch.arange(20, dtype=torch.int32, device="cuda").view(2, 10)
    Q = torch.randn((2, 8, 128), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(
        lib.TYPES[type_] if type_ != "e4m3" else torch.bfloat16)
    Q[0, 1, 3], Q[1, 5, 100], Q[1, 6] = math.nan, math.inf, -math.inf
    lens = torch.tensor([150, 99], dtype=torch.int32, device="cuda")
    lse = torch.empty((2, 8), device="cuda")
    O = PagedKV(kv, K, V, ke, ve).paged_attention(Q, tables, lens, lse_out=lse)
    bad = torch.zeros((2, 8), dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[1, 5] = bad[1, 6] = True
    assert O[bad].isnan().all() and lse[bad].isnan().all()
    fine = Q.clone()
    fine[bad] = 0
    ref = lib.attend(fine, K, V, ke, ve, tables, [150, 99])
    lib.assert_attends(O[~bad], lse[~bad], [x[~bad] for x in ref])


@pytest.mark.parametrize("type_", ["bf16", "f16"])
def test_an_infinite_value_under_a_small_weight(kv, type_):
    """Its column is infinite; NaN where the weight is so small that it counts for nothing (2^-33 of the largest in fp16).  No
    other column sees it."""
    from paper_2605_22718_b200 import PagedKV
    n, d = 40, 64
    for below, nan in ((20.0, False), (30.0, False), (40.0, type_ == "f16"), (200.0, True)):
        K, V, _, _ = lib.cache(type_, 3, 16, 1, d)
        K.zero_()
        K.view(-1, d)[7, 0] = 16.0
        V.view(-1, d)[20, 9] = math.inf
        Q = torch.zeros((1, 1, d), dtype=lib.TYPES[type_], device="cuda")
        Q[..., 0] = 1.0
        tables, lens = torch.arange(3, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda")
        O = PagedKV(kv, K, V).paged_attention(Q, tables, lens, softmax_scale=below * math.log(2) / 16)[0, 0]
        assert O[9].isnan() if nan else O[9] == math.inf, (below, O[9])
        rest = torch.arange(d, device="cuda") != 9
        want = V.view(-1, d)[:n].double()
        w = torch.softmax(K.view(-1, d)[:n, 0].double() * below * math.log(2) / 16, 0)
        want = (w[:, None] * want)[:, rest].sum(0)
        assert ((O[rest].double() - want).abs() <= 2 * lib.HALF_STEP[O.dtype] * want.abs() + 2.0 ** -20).all()
