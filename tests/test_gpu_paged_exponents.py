"""wk_paged_attention on 8-bit caches whose arrays of exponents are not a multiple of four bytes long."""
import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


@pytest.mark.parametrize("n_pages,page,heads", [(1, 1, 1), (1, 2, 1), (1, 3, 1), (1, 5, 1), (3, 1, 1), (2, 3, 1), (1, 1, 3), (5, 7, 3), (3, 33, 5), (9, 11, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_the_last_bytes_of_the_exponents(kv, n_pages, page, heads, d):
    """Every byte is that of its own row, the array's last ones too, whatever lies behind them."""
    from paper_2605_22718_b200 import PagedKV
    n = n_pages * page
    K, V, ke, ve = lib.cache("e4m3", n_pages, page, heads, d, seed=n)
    behind = []
    for e in (ke, ve):
        room = torch.full((e.numel() + 4,), 255, dtype=torch.uint8, device="cuda")
        room[:e.numel()] = e.view(-1)
        behind.append(room[:e.numel()].view(e.shape))
    Q = torch.randn((1, heads * 2, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    tables = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    lse = torch.empty((1, heads * 2), device="cuda")
    for window in (0, 1):                                   # all, and only the first page's last token
        O = PagedKV(kv, K, V, *behind).paged_attention(Q, tables, lens, window=window, lse_out=lse)
        lib.assert_attends(O, lse, lib.attend(Q, K, V, ke, ve, tables, [n], window))
    last = torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
    O = PagedKV(kv, K, V, *behind).paged_attention(Q, last, torch.tensor([page], dtype=torch.int32, device="cuda"), window=1, lse_out=lse)
    lib.assert_attends(O, lse, lib.attend(Q, K, V, ke, ve, last, [page], 1))
    assert kv.poll_status() == (0, 0)
