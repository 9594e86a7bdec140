"""Every token of wk_paged_attention counts once: with keys of zero all weights are equal, so that lse is the logarithm of how many tokens
were attended, and outputs count the tokens whose values are marked."""
import math

import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu
MARK = 64.0


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


def positions(n, window, sink):
    t = torch.arange(n, device="cuda")
    return t if not window else t[(t < sink) | (t >= n - window)]


def marks(t, head, d):
    """The column in which token t has its mark, or -1: of every eight tokens in a row one is marked, so of every step at least two;
    the columns take turns."""
    return torch.where((t + 3 * head) % 8 == 0, (t // 8) % d, -1)


def counted(kv, type_, d, heads, kv_heads, lens, window=0, sink=0, page=16, lose=None):
    """(O, lse, the counts that O stands for, tokens attended).  Whatever is not to be attended is NaN."""
    from paper_2605_22718_b200 import PagedKV
    dt = lib.TYPES[type_]
    have = [-(-max(n, 0) // page) for n in lens]
    n_pages = sum(have) + 1
    K, V = (torch.empty((n_pages, page, kv_heads, d), dtype=dt, device="cuda") for _ in range(2))
    for x in (K, V):
        x.view(torch.uint8 if type_ == "e4m3" else torch.int16).fill_(0x7f if type_ == "e4m3" else 0x7fff)
    exps = [None, None]
    if type_ == "e4m3":
        exps = [torch.full((n_pages, kv_heads, page), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(len(lens))).int()
    tables = torch.full((len(lens), max(have) + 2), 10 ** 9, dtype=torch.int32)
    counts = torch.zeros((len(lens), kv_heads, d), dtype=torch.float64, device="cuda")
    shown, at = [], 0
    for r, n in enumerate(lens):
        tables[r, :have[r]] = ids[at:at + have[r]]
        at += have[r]
        t = positions(max(n, 0), window, sink)
        shown.append(len(t))
        if not len(t):
            continue
        where, off = tables[r].cuda().long()[t // page], t % page
        for h in range(kv_heads):
            col = marks(t, h, d)
            row = torch.zeros((len(t), d), device="cuda")
            has = (col >= 0).nonzero().squeeze(1)
            power = torch.ones(len(t), device="cuda")
            if type_ == "e4m3":                       # marks of one size, stored under powers of 1 to 4
                byte = 127 + (t // 3) % 3
                power = torch.pow(2.0, byte.double() - 127).float()
                exps[1][where, h, off] = byte.to(torch.uint8)
                exps[0][where, h, off] = (100 + t % 50).to(torch.uint8)
            row[has, col[has]] = MARK / power[has]
            K[where, off, h] = torch.zeros((), device="cuda").to(dt)
            V[where, off, h] = row.to(dt)
            counts[r, h].scatter_add_(0, col[has], torch.ones(len(has), dtype=torch.float64, device="cuda"))
    if lose:
        lose(tables, K, V)
    g = torch.Generator(device="cuda").manual_seed(1)
    Q = torch.randn((len(lens), heads, d), generator=g, device="cuda").to(dt if type_ != "e4m3" else torch.float16)
    lse = torch.full((len(lens), heads), 77.0, device="cuda")
    O = torch.full_like(Q, 55)
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    PagedKV(kv, K, V, *exps).paged_attention(Q, tables.cuda(), dev, window=window, sink=sink, O=O, lse_out=lse)
    return O, lse, counts, shown


def check(kv, type_, d, heads, kv_heads, lens, window=0, sink=0, page=16, **kw):
    """Weights are powers of two, so products and their sums are exact; of n equal weights the sums are, too, up to 2^24.  What is left: joining
    at most 296 pieces twice (a factor off by 2^-22 and a sum off by 2^-24 of it each), a division (2^-22), logarithms off by 2^-21 and
    rounded to steps of 2^-19 at most, in pieces, then joined twice; O is rounded once."""
    O, lse, counts, shown = counted(kv, type_, d, heads, kv_heads, lens, window, sink, page, **kw)
    assert kv.poll_status() == (0, 0)
    half = lib.HALF_STEP[O.dtype]
    joins = 2 * (2.0 ** -22 + 296 * 2.0 ** -24) + 2.0 ** -22 + 3 * math.log(2) * (2.0 ** -21 + 2.0 ** -20)
    for r, n in enumerate(shown):
        if lens[r] < 0:
            assert (O[r] == 55).all() and (lse[r] == 77).all()
            continue
        if n == 0:
            assert (O[r] == 0).all() and (lse[r] == -math.inf).all()
            continue
        off = (lse[r].double() - math.log(n)).abs().max().item()
        assert off <= joins + 2.0 ** -20, (r, n, off)
        want = (counts[r] * MARK / n).repeat_interleave(heads // kv_heads, 0)
        bad = (O[r].double() - want).abs() > (half + joins) * want + 2.0 ** -25
        assert not bad.any(), (r, n, bad.nonzero()[:5].tolist(), O[r][bad][:5], want[bad][:5])


CASES = [
    # long runs: neighbouring heads side by side, several units to a kv head, windows
    ("e4m3", 128, 16, 8, [90000, 41111, 1, 0, 7000], 0, 0), ("e4m3", 128, 12, 12, [60001, 33333], 0, 0), ("e4m3", 64, 5, 5, [400000], 0, 0),
    ("f16", 64, 40, 40, [9999, 20000, 5, 8192], 0, 0), ("bf16", 128, 80, 4, [50000, 20003], 0, 0), ("bf16", 128, 66, 2, [90001, 0, 30], 0, 0),
    ("e4m3", 128, 8, 8, [110000, 90000], 80000, 77), ("bf16", 128, 8, 8, [90000, 33], 0, 0), ("f16", 128, 20, 1, [120000], 100000, 3),
    ("bf16", 64, 16, 16, [30000] * 5, 0, 0), ("e4m3", 64, 33, 1, [100000, 77], 0, 0), ("f16", 64, 16, 8, [70001, -1, 69999], 0, 0),
    # ragged batches, short ones, single tokens
    ("bf16", 128, 32, 8, [97 + 311 * i % 7000 for i in range(20)], 0, 0), ("f16", 64, 16, 16, [1 + 37 * i % 300 for i in range(120)], 0, 0),
    ("e4m3", 128, 40, 8, [1000 + 777 * i % 9000 for i in range(11)], 0, 0), ("bf16", 128, 12, 12, [880], 0, 0), ("bf16", 128, 4, 4, [1] * 37, 0, 0),
    ("f16", 64, 32, 8, [55] * 20, 0, 0), ("e4m3", 64, 8, 8, [205] * 31, 0, 0), ("bf16", 128, 4, 1, [120, 136, 8] * 20, 0, 0),
    ("bf16", 64, 20, 1, [90] * 16, 0, 0), ("bf16", 128, 28, 4, [500 + 997 * i % 20000 for i in range(24)], 1760, 880),
    ("f16", 128, 3, 3, [-1, 40, 0, 17, -1] * 12 + [-1] * 50, 0, 0), ("e4m3", 128, 16, 16, [256, 257, 31] * 11, 0, 0),
    ("f16", 64, 2, 1, [13 * i % 40 - 1 for i in range(9000)], 0, 0),
    ("f16", 128, 9, 1, [3000], 16, 0), ("e4m3", 64, 4, 4, [0, 1, 2, 63, 64, 65, 127, 128, 129], 0, 0),
]


@pytest.mark.parametrize("type_,d,heads,kv_heads,lens,window,sink", CASES)
@pytest.mark.parametrize("page", [16, 100])
def test_every_token_counts_once(kv, type_, d, heads, kv_heads, lens, window, sink, page):
    check(kv, type_, d, heads, kv_heads, lens, window, sink, page)


@pytest.mark.parametrize("type_,d,heads,kv_heads,lens,window,sink", CASES[:4] + CASES[12:16])
def test_lost_tokens_would_be_seen(kv, type_, d, heads, kv_heads, lens, window, sink):
    """The tests' own eyes: a page taken from a table somewhere in the longest request, and one whose values read as zeros, are both noticed."""
    longest = max(range(len(lens)), key=lambda r: lens[r])
    place = lens[longest] // 16 // 3

    def a_page(tables, K, V):
        tables[longest, place] = -1

    def its_values(tables, K, V):
        V[tables[longest, place]] = torch.zeros((), device="cuda").to(V.dtype)
    for lose in (a_page, its_values):
        with pytest.raises(AssertionError):
            check(kv, type_, d, heads, kv_heads, lens, window, sink, lose=lose)
