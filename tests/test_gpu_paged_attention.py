"""wk_paged_attention against the formula in 64 bits: types, head layouts, ragged lengths, windows, pages, strides, refusals of the device."""
import math

import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


def queries(B, H, d, dtype, seed=11, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn((B, H, d), generator=g, device="cuda")).to(dtype)


def setup(type_, lens, heads, kv_heads, d, page, layout="tokens", q16=None, seed=0, window=0, sink=0, dirty=True, size=1.0):
    """Inputs of a call; whatever it may not look at is NaN, and table places past a request's pages are ids out of range."""
    max_pages = max(1, max(-(-max(n, 0) // page) for n in lens)) + 1
    n_pages = sum(-(-max(n, 0) // page) for n in lens) + 2
    K, V, ke, ve = lib.cache(type_, n_pages, page, kv_heads, d, seed, layout)
    tables = lib.tables_for(lens, page, n_pages, max_pages, seed)
    if dirty:
        lib.poison(K, V, ke, ve, tables.cpu(), lens, window, sink)
    qt = q16 or (lib.TYPES[type_] if type_ != "e4m3" else torch.bfloat16)
    return K, V, ke, ve, tables, torch.tensor(lens, dtype=torch.int32, device="cuda"), queries(len(lens), heads, d, qt, seed + 1, size)


def call(kv, K, V, ke, ve, tables, lens, Q, **kw):
    from paper_2605_22718_b200 import PagedKV
    lse = torch.full(Q.shape[:2], 77.0, dtype=torch.float32, device="cuda")
    O = torch.full(Q.shape, 55.0, dtype=Q.dtype, device="cuda")
    got = PagedKV(kv, K, V, ke, ve).paged_attention(Q, tables, lens, O=O, lse_out=lse, **kw)
    assert got is O
    return O, lse


def check(kv, s, **kw):
    K, V, ke, ve, tables, lens, Q = s
    O, lse = call(kv, K, V, ke, ve, tables, lens, Q, **kw)
    lib.assert_attends(O, lse, lib.attend(Q, K, V, ke, ve, tables, lens.tolist(), kw.get("window", 0), kw.get("sink", 0),
                                          kw.get("softmax_scale", 0.0)))
    assert kv.poll_status() == (0, 0)
    return O, lse


EDGES = [0, 1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 257, 300]


@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("share", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 20, 33])
def test_every_length_near_a_tile_and_every_sharing(kv, type_, d, share):
    kv_heads = 2 if share > 4 else 3
    check(kv, setup(type_, EDGES, kv_heads * share, kv_heads, d, 16, seed=share))


@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("page", [1, 3, 8, 24, 64, 100, 1000])
@pytest.mark.parametrize("layout", ["tokens", "heads", "paired"])
def test_pages_and_layouts(kv, type_, page, layout):
    check(kv, setup(type_, [0, 1, 5, 99, 100, 101, 777], 10, 5, 128 if page != 24 else 64, page, layout, seed=page))


@pytest.mark.parametrize("lens,heads,kv_heads", [
    ([1], 1, 1), ([2], 12, 12), ([5000], 1, 1), ([5000], 40, 8), ([4999], 20, 1), ([3001, 1], 16, 1), ([1] * 300, 4, 2),
    ([(37 * i) % 90 for i in range(1100)], 3, 3), ([2000, 0, 3, 0, 1999] * 3, 8, 8), ([0] * 9, 4, 4), ([1200] * 40, 80, 40),
])
@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
def test_batches(kv, type_, lens, heads, kv_heads):
    check(kv, setup(type_, lens, heads, kv_heads, 128, 16, seed=len(lens), dirty=len(lens) < 400))


@pytest.mark.parametrize("q16", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [2.0 ** -12, 1.0, 2.0 ** 10])
def test_queries_of_both_types_on_8_bits(kv, q16, size):
    """Query rows of any size: a power of two per row brings them into fp16 and is taken out of the logits again."""
    s = list(setup("e4m3", [0, 1, 40, 333], 12, 4, 128, 16, q16=q16, size=size))
    if size > 1:
        s[2].sub_(14)                                  # keys so small that the logits are ordinary
        s[2].clamp_(min=1)
        lib.poison(*s[:4], s[4].cpu(), s[5].tolist())
    s[6][:, 3] = 0
    s[6][:, 4, 5:] *= 2.0 ** -6
    check(kv, s)


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (16, 0), (5, 3), (64, 16), (100, 33), (129, 1), (1000, 1000), (2 ** 31 - 1, 5)])
@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
def test_windows(kv, type_, window, sink):
    """Tokens outside the window are NaN, and pages that lie outside altogether are ids out of range."""
    lens = [0, 1, 2, 15, 16, 17, 100, 133, 134, 135, 700]
    s = setup(type_, lens, 8, 4, 128, 16, window=window, sink=sink)
    for b, n in enumerate(lens):
        seen = {t // 16 for t in lib.visible(n, window, sink)}
        for i in range(s[4].shape[1]):
            if i not in seen:
                s[4][b, i] = -3
    check(kv, s, window=window, sink=sink)


def test_padded_rows_stay_as_they_are(kv):
    K, V, ke, ve, tables, lens, Q = setup("bf16", [40, -1, 0, -5, 100, -1], 4, 4, 128, 16)
    O, lse = call(kv, K, V, ke, ve, tables, lens, Q)
    out = lens < 0
    assert (O[out] == 55).all() and (lse[out] == 77).all()
    assert (O[2] == 0).all() and (lse[2] == -math.inf).all()
    ref = lib.attend(Q, K, V, ke, ve, tables, lens.tolist())
    lib.assert_attends(O[~out], lse[~out], [x[~out] for x in ref])
    only = torch.full((6,), -1, dtype=torch.int32, device="cuda")
    O, lse = call(kv, K, V, ke, ve, tables, only, Q)
    assert (O == 55).all() and (lse == 77).all() and kv.poll_status() == (0, 0)


@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
def test_pages_that_are_not_there(kv, type_):
    from paper_2605_22718_b200 import WK_DEV_BAD_SLOT
    s = setup(type_, [100, 64, 200, 16], 8, 2, 128, 16, dirty=False)
    tables = s[4]
    tables[0, 2] = tables[2, 0] = tables[2, 12] = tables[3, 0] = -1         # the last request has nothing left
    lib.poison(*s[:4], tables.cpu(), s[5].tolist())
    O, lse = check(kv, s)
    assert (O[3] == 0).all() and (lse[3] == -math.inf).all()
    tables[1, 1], tables[0, 6], tables[2, 5] = s[0].shape[0], -2, 2 ** 31 - 1
    O, lse = call(kv, *s)
    lib.assert_attends(O, lse, lib.attend(s[6], *s[:4], tables, s[5].tolist()))
    assert kv.poll_status()[1] == WK_DEV_BAD_SLOT


def test_a_length_beyond_the_table(kv):
    from paper_2605_22718_b200 import WK_DEV_BAD_SLOT
    s = setup("bf16", [64, 48], 4, 2, 128, 16, dirty=False)
    wide = s[4]
    s = (*s[:4], wide[:, :3].contiguous(), torch.tensor([2 ** 31 - 1, 49], dtype=torch.int32, device="cuda"), s[6])
    O, lse = call(kv, *s)
    lib.assert_attends(O, lse, lib.attend(s[6], *s[:4], s[4], [48, 48]))
    assert kv.poll_status()[1] == WK_DEV_BAD_SLOT


@pytest.mark.parametrize("type_,logit", [("bf16", 60.0), ("f16", 60.0), ("e4m3", 60.0), ("bf16", 3000.0)])
def test_logits_that_rise_fall_and_tower(kv, type_, logit):
    """The running maximum: keys along the query with rising, falling and single large coefficients."""
    n, d = 700, 128
    K, V, ke, ve, tables, lens, Q = setup(type_, [n, n, n], 6, 3, d, 16, dirty=False)
    Q.copy_(torch.sign(Q))
    coef = torch.linspace(0, 1, n, device="cuda")
    shapes = [coef, coef.flip(0), torch.where(torch.arange(n, device="cuda") == 433, 1.0, 0.01)]
    for b in range(3):
        ids = tables[b].long()[torch.arange(n, device="cuda") // 16]
        off = torch.arange(n, device="cuda") % 16
        k = shapes[b][:, None, None] * Q[b, 0::2].float()[None] * logit / d ** 0.5
        if type_ == "e4m3":
            ke.transpose(1, 2)[ids, off] = 121
            k = k * 64
        K[ids, off] = k.to(K.dtype)
    check(kv, (K, V, ke, ve, tables, lens, Q))


@pytest.mark.parametrize("type_", ["bf16", "f16"])
def test_values_that_are_not_finite(kv, type_):
    """A logit of NaN or +inf spoils its head's row and no other; a key with all logits -inf leaves no weight; V's stay in their column."""
    K, V, ke, ve, tables, lens, Q = setup(type_, [50, 50, 50, 50], 4, 4, 128, 16)
    Q.copy_(Q.abs() + 0.5)
    at = lambda b, t: (int(tables[b, t // 16]), t % 16)  # noqa: E731
    K[at(0, 17)][1, 5] = math.nan
    K[at(1, 49)][2, 0] = math.inf
    for t in range(50):
        K[at(2, t)][0, 127] = -math.inf
    V[at(3, 3)][3, 64] = math.inf
    V[at(3, 3)][3, 65] = math.nan
    O, lse = check(kv, (K, V, ke, ve, tables, lens, Q))
    assert O[0, 1].isnan().all() and lse[0, 1].isnan() and O[1, 2].isnan().all() and not O[0, 0].isnan().any()
    assert (O[2, 0] == 0).all() and lse[2, 0] == -math.inf
    assert O[3, 3].isinf().sum() == 1 and O[3, 3].isnan().sum() == 1


def test_scales_and_strides(kv):
    K, V, ke, ve, tables, lens, Q = setup("bf16", [130, 7, 64], 12, 4, 128, 16)
    check(kv, (K, V, ke, ve, tables, lens, Q), softmax_scale=0.5)
    fused = torch.randn((3, 20, 128), device="cuda").to(torch.bfloat16)     # queries beside keys and values in one row
    check(kv, (K, V, ke, ve, tables, lens, fused[:, :12]))
    wide = torch.full((3, tables.shape[1] + 5), 10 ** 9, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + tables.shape[1]] = tables
    check(kv, (K, V, ke, ve, wide[:, 2:2 + tables.shape[1]], lens, Q))
    from paper_2605_22718_b200 import PagedKV
    O = PagedKV(kv, K, V).paged_attention(Q, tables, lens)                   # no lse, O allocated
    lse = torch.empty((3, 12), device="cuda")
    ref = lib.attend(Q, K, V, None, None, tables, lens.tolist())
    again = Q.clone()
    assert PagedKV(kv, K, V).paged_attention(again, tables, lens, O=again, lse_out=lse) is again      # O over Q
    assert torch.equal(O, again)
    lib.assert_attends(O, lse, ref)


@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
def test_a_cache_past_32_bits(kv, type_):
    """Pages beyond 4 GB of a cache: the first, the last and those around 2^31 and 2^32."""
    from paper_2605_22718_b200 import PagedKV
    page, heads, d = 16, 8, 128
    row = heads * d * (2 if type_ == "bf16" else 1)
    n_pages = (9 << 30) // (page * row)
    dt = lib.TYPES[type_]
    K, V = (torch.empty((n_pages, page, heads, d), dtype=dt, device="cuda") for _ in range(2))
    ke, ve = (torch.full((n_pages, heads, page), 120, dtype=torch.uint8, device="cuda") if type_ == "e4m3" else None for _ in range(2))
    per = 1 << 31
    ids = [0, per // (page * row) - 1, per // (page * row), 2 * per // (page * row) - 1, 2 * per // (page * row),
           4 * per // (page * row) - 1, 4 * per // (page * row), n_pages - 1]
    g = torch.Generator(device="cuda").manual_seed(3)
    for x in (K, V):
        x[ids] = (torch.randn((8, page, heads, d), generator=g, device="cuda") * (1 if type_ == "bf16" else 100)).to(dt)
    tables = torch.tensor([ids], dtype=torch.int32, device="cuda")
    Q = queries(1, 16, d, torch.bfloat16)
    lens = torch.tensor([125], dtype=torch.int32, device="cuda")
    lse = torch.empty((1, 16), device="cuda")
    O = PagedKV(kv, K, V, ke, ve).paged_attention(Q, tables, lens, lse_out=lse)
    lib.assert_attends(O, lse, lib.attend(Q, K, V, ke, ve, tables, [125]))


def test_two_calls_give_the_same_bits(kv):
    s = setup("bf16", [3000, 17, 900, 1], 16, 4, 128, 16)
    first = [x.clone() for x in call(kv, *s)]
    for _ in range(5):
        assert all(torch.equal(x, y) for x, y in zip(first, call(kv, *s)))


def test_many_calls_with_changing_batches_share_the_scratch(kv):
    """Counters are back at zero after every call, whatever was shared between which blocks."""
    for i, lens in enumerate([[4000], [1, 2, 3], [700] * 33, [0, -1, 5000, 3], [16] * 200, [4000]]):
        s = setup("bf16", lens, 8, 4, 64 if i % 2 else 128, 16, seed=i)
        K, V, ke, ve, tables, dev, Q = s
        O, lse = call(kv, *s)
        keep = dev >= 0
        lib.assert_attends(O[keep], lse[keep], [x[keep] for x in lib.attend(Q, K, V, ke, ve, tables, lens)])


def test_refusals(kv):
    from paper_2605_22718_b200 import PagedKV, WkError, WK_ERR_ARG, WK_ERR_SHAPE
    K, V, ke, ve, tables, lens, Q = setup("bf16", [5, 6], 12, 4, 128, 16)
    c = PagedKV(kv, K, V)
    for status, args, kw in [
            (WK_ERR_SHAPE, (Q[:, :10].contiguous(), tables, lens), {}), (WK_ERR_ARG, (Q.half(), tables, lens), {}),
            (WK_ERR_ARG, (Q.float(), tables, lens), {}), (WK_ERR_ARG, (Q[..., :64], tables, lens), {}),
            (WK_ERR_ARG, (Q.cpu(), tables, lens), {}), (WK_ERR_ARG, (Q, tables.long(), lens), {}),
            (WK_ERR_ARG, (Q, tables, lens.long()), {}), (WK_ERR_ARG, (Q, tables[:1], lens), {}), (WK_ERR_ARG, (Q, tables, lens[:1]), {}),
            (WK_ERR_ARG, (Q, tables, lens), dict(O=Q.float())), (WK_ERR_ARG, (Q, tables, lens), dict(lse_out=Q)),
            (WK_ERR_ARG, (Q, tables, lens), dict(window=-1)), (WK_ERR_ARG, (Q, tables, lens), dict(softmax_scale=-0.5)),
            (WK_ERR_SHAPE, (Q, tables, lens), dict(scratch=torch.zeros(256, dtype=torch.uint8, device="cuda")[:0])),
            (WK_ERR_ARG, (Q.transpose(1, 2).contiguous().transpose(1, 2), tables, lens), {})]:
        with pytest.raises(WkError) as e:
            c.paged_attention(*args, **kw)
        assert e.value.status in (status, WK_ERR_ARG), (args, kw)
    assert c.paged_attention(Q[:0], tables[:0], lens[:0]).shape == (0, 12, 128)


@pytest.mark.parametrize("type_,d,heads,kv_heads,lens,window,sink", [
    ("e4m3", 128, 16, 8, [90000, 41111, 1, 0, 7000], 0, 0),          # neighbouring heads side by side, runs of a few hundred steps
    ("e4m3", 128, 12, 12, [60001, 33333], 0, 0),
    ("e4m3", 64, 5, 5, [400000], 0, 0),
    ("f16", 64, 40, 40, [9999, 20000, 5, 8192], 0, 0),               # five heads one after the other on each of eight lines
    ("bf16", 128, 80, 4, [50000, 20003], 0, 0),                      # two units share every kv head
    ("bf16", 128, 66, 2, [100001, 0, 30], 0, 0),                     # three do
    ("e4m3", 128, 8, 8, [150000, 90000], 100000, 77),
])
def test_long_runs(kv, type_, d, heads, kv_heads, lens, window, sink):
    check(kv, setup(type_, lens, heads, kv_heads, d, 64, seed=3, window=window, sink=sink, dirty=False), window=window, sink=sink)


@pytest.mark.parametrize("type_,d,heads,kv_heads,lens", [
    ("f16", 64, 32, 8, [55] * 20), ("e4m3", 64, 8, 8, [205] * 31), ("bf16", 128, 4, 4, [1] * 37), ("bf16", 128, 8, 2, [128, 0, 1, 129, 16, 17] * 9),
    ("bf16", 128, 4, 1, [120, 136, 8] * 40), ("e4m3", 128, 16, 16, [256, 257, 31] * 11), ("f16", 64, 3, 3, [300] * 77), ("bf16", 64, 20, 1, [90] * 16),
])
def test_short_runs(kv, type_, d, heads, kv_heads, lens):
    """So little work that every warp has a few steps: CTAs begin and end with short units."""
    check(kv, setup(type_, lens, heads, kv_heads, d, 16, seed=len(lens)))


def test_a_short_run_beside_rows_that_do_not_exist(kv):
    lens = ([-1, 40, 0, 17, -1] * 12) + [-1] * 300
    K, V, ke, ve, tables, dev, Q = setup("bf16", lens, 8, 4, 128, 16)
    O, lse = call(kv, K, V, ke, ve, tables, dev, Q)
    there = dev >= 0
    assert (O[~there] == 55).all() and (lse[~there] == 77).all()
    lib.assert_attends(O[there], lse[there], [x[there] for x in lib.attend(Q, K, V, ke, ve, tables, lens)])


def test_an_output_of_a_tensor_subclass(kv):
    from paper_2605_22718_b200 import PagedKV
    K, V, _, _, tables, lens, Q = setup("bf16", [33], 4, 4, 128, 16)
    O = torch.nn.Parameter(torch.empty_like(Q), requires_grad=False)
    assert PagedKV(kv, K, V).paged_attention(Q, tables, lens, O=O) is O
    assert torch.equal(O, PagedKV(kv, K, V).paged_attention(torch.nn.Parameter(Q, requires_grad=False), tables, lens))


def test_tables_with_room_for_more_than_31_bits_of_steps(kv):
    """3,000 requests whose tables could name 320,000 tokens each, 40 kv heads: more than one launch counts, so there are two."""
    from paper_2605_22718_b200 import PagedKV
    n, width = 3000, 20000
    lens = [(i * 7) % 40 - 1 for i in range(n)]
    n_pages = sum(-(-max(m, 0) // 16) for m in lens) + 1
    K, V, _, _ = lib.cache("f16", n_pages, 16, 40, 64)
    tables = torch.full((n, width), -7, dtype=torch.int32, device="cuda")
    tables[:, :4] = lib.tables_for(lens, 16, n_pages, 4)
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    Q = queries(n, 40, 64, torch.float16)
    lse = torch.full((n, 40), 77.0, device="cuda")
    O = torch.full_like(Q, 55)
    c = PagedKV(kv, K, V)
    before = kv.launch_count()
    c.paged_attention(Q, tables, dev, O=O, lse_out=lse)
    assert kv.launch_count() == before + 2
    some = torch.tensor([i for i in range(n) if i % 97 == 0 or i > n - 5 or 2676 < i < 2690], device="cuda")
    keep = some[dev[some] >= 0]
    ref = lib.attend(Q[keep], K, V, None, None, tables[keep], [lens[i] for i in keep.tolist()])
    lib.assert_attends(O[keep], lse[keep], ref)
    assert (O[dev < 0] == 55).all() and (lse[dev < 0] == 77).all() and kv.poll_status() == (0, 0)
    narrow = tables[:, :4].contiguous()          # the same with room for 64 tokens: one launch, the same rows
    again, lse2 = torch.full_like(Q, 55), torch.full_like(lse, 77.0)
    c.paged_attention(Q, narrow, dev, O=again, lse_out=lse2)
    assert kv.launch_count() == before + 3
    lib.assert_attends(again[keep], lse2[keep], ref)
