"""wk_paged_attention where softmax weights are far below the largest: tails that only together weigh something."""
import math

import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


def one_above_many(kv, type_, gap, n=20000, d=64, place=0, rows=1600):
    """O, lse of one key `gap` above n others, whose values are whole numbers and its own are zero.  So many requests over the same
    pages that no request is shared by warps: each meets the whole tail behind one reference."""
    from paper_2605_22718_b200 import PagedKV
    dt, page = lib.TYPES[type_], 64
    n_pages = -(-(n + 1) // page)
    K, V = (torch.zeros((n_pages, page, 1, d), dtype=torch.float32, device="cuda") for _ in range(2))
    values = (torch.arange(d, device="cuda") % 15 - 7).float()
    V.view(-1, d)[:n + 1] = values
    K.view(-1, d)[place, 0] = 16.0
    V.view(-1, d)[place] = 0
    exps = [torch.full((n_pages, 1, page), b, dtype=torch.uint8, device="cuda") if type_ == "e4m3" else None for b in (127, 119)]
    if type_ == "e4m3":
        V *= 2.0 ** 5                                              # codes of up to 224, 2^-8 each
        values = values * 2.0 ** -3
    Q = torch.zeros((rows, 1, d), dtype=torch.bfloat16 if type_ == "bf16" else torch.float16, device="cuda")
    Q[..., 0] = gap / 16.0
    assert Q[0, 0, 0].item() * 16.0 == gap
    tables = torch.arange(n_pages, dtype=torch.int32, device="cuda").repeat(rows, 1)
    lens = torch.full((rows,), n + 1, dtype=torch.int32, device="cuda")
    lse = torch.empty((rows, 1), device="cuda")
    O = PagedKV(kv, K.to(dt), V.to(dt), *exps).paged_attention(Q, tables, lens, softmax_scale=1.0, lse_out=lse)
    assert kv.poll_status() == (0, 0)
    return O.double(), lse.double(), values.double()


@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("gap", [9.0, 12.5, 17.0, 17.375, 19.0])
@pytest.mark.parametrize("place", [0, 7777, 20000])
def test_a_tail_far_below_one_key(kv, type_, gap, place):
    """Of n weights each is off by u of itself, or by 2^-32 of the largest where it is rounded to fp16's lowest steps; the exponential by 2^-22 and
    its argument by 2^-23 of its size, twice; sums over n values by n * 2^-23; O is rounded once more."""
    n = 20000
    O, lse, values = one_above_many(kv, type_, gap, n=n, place=place)
    w = math.exp(-gap)
    total = 1 + n * w
    want = n * w / total * values
    u = 2.0 ** -8 if type_ == "bf16" else 2.0 ** -11
    rel = u + 2.0 ** -22 + 2 * gap * 2.0 ** -23 + 2 * n * 2.0 ** -23
    tol = rel * want.abs() + (0 if type_ == "bf16" else n * 2.0 ** -32 / total * values.abs())
    tol = tol + lib.HALF_STEP[torch.bfloat16 if type_ == "bf16" else torch.float16] * (want.abs() + tol) + 2.0 ** -25
    assert ((O - want).abs() <= tol).all(), ((O - want).abs() / tol).max().item()
    want = gap + math.log(total)
    assert (lse - want).abs().max().item() <= 2 * gap * 2.0 ** -22 + 2.0 ** -21 + n * 2.0 ** -23 + want * 2.0 ** -22


@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** 27, 2.0 ** 30])
def test_logits_beyond_what_their_steps_resolve(kv, type_, size):
    """Logits that rise by one step of 32 bits at a time, some of them far larger than softmax can tell apart: weights stay finite, and every
    output lies between the values that it is a mean of."""
    from paper_2605_22718_b200 import PagedKV
    n, d, page = 700, 64, 16
    n_pages = -(-n // page)
    dt = lib.TYPES[type_]
    K, V = (torch.zeros((n_pages * page, 1, d), dtype=torch.float32, device="cuda") for _ in range(2))
    t = torch.arange(n, device="cuda").float()
    K[:n, 0, 0], K[:n, 0, 1] = 256.0, t // 8 if type_ != "e4m3" else t // 88
    V[:n, 0] = (t % 5 + 1)[:, None]
    K, V = (x.view(n_pages, page, 1, d).to(dt) for x in (K, V))
    exps = [torch.full((n_pages, 1, page), 127, dtype=torch.uint8, device="cuda") if type_ == "e4m3" else None for _ in range(2)]
    Q = torch.zeros((3, 2, d), dtype=torch.bfloat16 if type_ == "bf16" else torch.float16, device="cuda")
    Q[..., 0], Q[..., 1] = 1.0, 2.0 ** -15                          # 256 rises by 2^-15
    tables = torch.arange(n_pages, dtype=torch.int32, device="cuda").repeat(3, 1)
    lens = torch.tensor([n, 350, 9], dtype=torch.int32, device="cuda")
    lse = torch.empty((3, 2), device="cuda")
    O = PagedKV(kv, K, V, *exps).paged_attention(Q, tables, lens, softmax_scale=size / 256.0 / math.log2(math.e), lse_out=lse)
    assert kv.poll_status() == (0, 0) and torch.isfinite(O).all() and torch.isfinite(lse).all()
    assert (O >= 0.99).all() and (O <= 5.05).all()


@pytest.mark.parametrize("size", [2.0 ** 120, 2.0 ** 127, 2.0 ** -60, 2.0 ** -100])
def test_values_of_any_size_in_8_bits(kv, size):
    """Rows of values near the largest and far below one, stored in 8 bits, under logits that rise slowly."""
    from paper_2605_22718_b200 import PagedKV
    n, d, page = 100, 64, 16
    c = PagedKV.empty(kv, 7, page, 1, d, torch.float8_e4m3fn)
    K = torch.zeros((n, 1, d), dtype=torch.bfloat16, device="cuda")
    K[..., 0] = (torch.arange(n, device="cuda") / 16.0)[:, None]
    V = (size * (1 + torch.arange(n, device="cuda")[:, None, None] % 7 / 8.0)).expand(n, 1, d).to(torch.bfloat16).contiguous()
    c.page_store(K, V, torch.arange(n, dtype=torch.int32, device="cuda"))
    Q = torch.zeros((1, 1, d), dtype=torch.bfloat16, device="cuda")
    Q[..., 0] = 1
    tables = torch.arange(7, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    O = c.paged_attention(Q, tables, lens, softmax_scale=1.0).double()
    ks = c.K.view(-1, d)[:n, 0].double() * torch.pow(2.0, c.K_exp.view(-1)[:n].double() - 127)
    vs = c.V.view(-1, d)[:n, 0].double() * torch.pow(2.0, c.V_exp.view(-1)[:n].double() - 127)
    want = (torch.softmax(ks, 0) * vs).sum()
    # weights off by half a step of fp16, exponentials and sums of 100 values by 2^-15 together, the output by half a step of bf16
    assert ((O - want).abs() <= (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -14) * want).all(), (O / want).max().item()
    assert kv.poll_status() == (0, 0)


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** -20, 2.0 ** -14, 1.0, 300.0])
@pytest.mark.parametrize("d,page,n", [(64, 16, 100), (128, 16, 333), (128, 5, 33)])
@pytest.mark.parametrize("signed", [False, True])
def test_rows_of_zeros_beside_small_values_in_8_bits(kv, size, d, page, n, signed):
    """A row of zeros is stored with the power 1: it lies far above the power of small values, and has nothing to add to them."""
    from paper_2605_22718_b200 import PagedKV
    n_pages = -(-n // page)
    c = PagedKV.empty(kv, n_pages, page, 2, d, torch.float8_e4m3fn)
    g = torch.Generator(device="cuda").manual_seed(n)
    K = torch.randn((n, 2, d), generator=g, device="cuda").to(torch.bfloat16)
    V = (size * (1 + torch.rand((n, 2, d), generator=g, device="cuda"))).to(torch.bfloat16)
    V[::7, 0] = 0
    V[n - 1, 1] = 0
    if signed:
        V *= torch.where(torch.arange(n, device="cuda") % 2 == 0, 1, -1)[:, None, None]     # zeros of either sign
        V[..., 0] = V[..., 0].abs()
    c.page_store(K, V, torch.arange(n, dtype=torch.int32, device="cuda"))
    if n > 30:
        V[28, 1] = 0                                            # zeros under another power: a cache that is written otherwise
        c.V.view(-1, 2, d).view(torch.uint8)[28, 1] = 0
    Q = torch.randn((1, 8, d), generator=g, device="cuda").to(torch.float16)
    tables = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    O = c.paged_attention(Q.to(torch.bfloat16), tables, lens).double()
    assert torch.equal((c.V_exp.transpose(1, 2).reshape(-1, 2)[:n] == 127)[::7, 0], torch.ones((n + 6) // 7, dtype=torch.bool, device="cuda"))
    rows = lambda x, e: x.reshape(-1, 2, d)[:n].double() * torch.pow(2.0, e.transpose(1, 2).reshape(-1, 2)[:n].double() - 127)[..., None]  # noqa: E731
    k, v = rows(c.K, c.K_exp), rows(c.V, c.V_exp)
    q = Q.to(torch.bfloat16).double().view(2, 4, d)
    logits = torch.einsum("hgd,nhd->hgn", q, k) / d ** 0.5
    p = torch.softmax(logits, -1)
    want = torch.einsum("hgn,nhd->hgd", p, v).reshape(1, 8, d)
    mags = torch.einsum("hgd,nhd->hgn", q.abs(), k.abs()).amax() / d ** 0.5
    # per weight: half a step of fp16, what a logit is off by (d products in 32 bits), the exponential; sums of n values; bf16
    rel = 2.0 ** -11 + 2 * ((d + 4) * 2.0 ** -23 * mags + 2.0 ** -22 * logits.abs().amax()) + 2.0 ** -22 + 2 * (n + 16) * 2.0 ** -23
    heavy = torch.einsum("hgn,nhd->hgd", p, v.abs()).reshape(1, 8, d)
    # weights (times their row's power) below 2^-14 of 2^7 times the largest: off by 2^-32 of that, times codes of up to 448
    ve = torch.where(v.abs().amax(-1) > 0, torch.pow(2.0, c.V_exp.transpose(1, 2).reshape(-1, 2)[:n].double() - 127), 0.0)
    low = n * 2.0 ** -32 * 448 * (p * ve.t()[:, None]).amax(-1).reshape(1, 8, 1)
    tol = rel * heavy + low
    tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert ((O - want).abs() <= tol).all(), ((O - want).abs() / tol).max().item()
    assert kv.poll_status() == (0, 0)
