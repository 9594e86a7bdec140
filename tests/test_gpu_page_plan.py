"""wk_page_plan against one request after the other: slots, starts, lengths, tables, ring and state are whole numbers and equal."""
import random

import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


def gpu(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Case:
    """Lists of a plan's inputs; pages of requests and of the ring are distinct."""

    def __init__(self, rng, lens, new, page, spare, max_pages=None, head=None, missing=0):
        up = lambda v: -(-v // page) if v > 0 else 0  # noqa: E731
        self.page, self.lens, self.new = page, list(lens), list(new)
        held = sum(up(n) for n in lens)
        self.n_pages = held + spare + missing          # missing: pages that nobody has (neither free nor held)
        ids = list(range(self.n_pages))
        rng.shuffle(ids)
        self.max_pages = max_pages or max(1, max(up(max(n, 0) + max(m, 0)) for n, m in zip(lens, new)))
        self.tables, at = [], 0
        for n in lens:
            self.tables.append(ids[at:at + up(n)] + [-7] * (self.max_pages - up(n)))
            at += up(n)
        self.head = rng.randrange(self.n_pages) if head is None else head
        self.ring = [-9] * self.n_pages
        for i in range(spare):
            self.ring[(self.head + i) % self.n_pages] = ids[at + i]
        self.count = spare
        self.most = sum(max(0, m) for m in new)

    def check(self, kv, in_place=True, wide=0):
        from paper_2605_22718_b200 import PagedKV
        ref = lib.plan(self.lens, self.new, self.tables, self.ring, self.head, self.count, self.page, self.most)
        c = PagedKV(kv, n_pages=self.n_pages, page_tokens=self.page)
        kv.poll_status()
        lens, ring, state = gpu(self.lens), gpu(self.ring), gpu([self.head, self.count, 0, 0])
        tables = gpu([t + [-5] * wide for t in self.tables])
        out = {} if in_place else dict(lens_out=torch.empty_like(lens), state_out=torch.empty_like(state))
        view = tables[:, :self.max_pages]
        slots, starts = c.page_plan(lens, gpu(self.new), view, ring, state, self.most, **out)
        flags = kv.poll_status()[1]
        if not in_place:
            assert lens.tolist() == self.lens and state.tolist() == [self.head, self.count, 0, 0]
        assert starts.tolist() == ref["starts"]
        assert slots.tolist() == ref["slots"]
        assert out.get("lens_out", lens).tolist() == ref["lens"]
        assert out.get("state_out", state).tolist() == ref["state"]
        assert view.tolist() == ref["tables"] and (tables[:, self.max_pages:] == -5).all()
        assert ring.tolist() == ref["ring"]
        from paper_2605_22718_b200 import WK_DEV_BAD_SLOT, WK_DEV_POOL_FULL
        assert flags == (WK_DEV_POOL_FULL if ref["full"] else 0) | (WK_DEV_BAD_SLOT if ref["bad"] else 0)
        return ref


@pytest.mark.parametrize("lens,new,page", [
    ([0], [1], 16), ([0], [0], 16), ([16], [1], 16), ([15], [1], 16), ([15], [2], 16), ([0], [5000], 16), ([3], [-1], 16),
    ([7], [9], 1), ([0, 5, 16, 17, 31, 32], [1, 1, 1, 1, 1, 1], 16), ([10, -1, 40, -1], [4, 0, -1, 0], 16),
    ([0, 0, 0], [100, 0, 33], 24), ([33, 64, 65], [-1, -1, -1], 32), ([0], [1 << 17], 128),
    ([5, 6, 7], [0, 0, 0], 4),
])
@pytest.mark.parametrize("in_place", [True, False])
def test_small_plans(kv, lens, new, page, in_place):
    Case(random.Random(1), lens, new, page, spare=2000 if max(new) < 6000 else 1100).check(kv, in_place)


@pytest.mark.parametrize("seed", range(12))
def test_random_plans(kv, seed):
    rng = random.Random(seed)
    n = rng.choice([1, 2, 33, 700, 1023, 1025, 2500, 4096])
    page = rng.choice([1, 4, 16, 24, 64])
    lens = [rng.choice([0, -1, rng.randrange(300)]) for _ in range(n)]
    new = [0 if l < 0 else rng.choice([1, 1, 1, 0, -1, rng.randrange(1, 60)]) for l in lens]
    c = Case(rng, lens, new, page, spare=sum(max(0, v) for v in new) + rng.randrange(50), missing=rng.randrange(9))
    c.check(kv, in_place=seed % 2 == 0, wide=seed % 3)


@pytest.mark.parametrize("spare", [0, 1, 5, 6, 7, 60])
def test_too_few_pages(kv, spare):
    """Requests are served in order as far as the pages go; one that needs none is always served."""
    lens, new = [16, 3, 0, 15, 40, 0, 1], [16, 2, 64, 1, 30, 1, 15]
    ref = Case(random.Random(3), lens, new, 16, spare).check(kv)
    assert ref["full"] == (spare < 8)
    assert ref["lens"][1] == 5 and ref["lens"][6] == 16


def test_tables_and_slot_lists_without_room(kv):
    ref = Case(random.Random(4), [10, 30, 32], [30, 3, 1], 16, spare=10, max_pages=2).check(kv)
    assert ref["lens"] == [10, 30, 32] and ref["full"]
    c = Case(random.Random(4), [1, 2, 3, 4], [5, 5, 5, 5], 16, spare=10)
    c.most = 12                                     # the third request's rows reach past the list
    ref = c.check(kv)
    assert ref["lens"] == [6, 7, 3, 4] and ref["starts"] == [0, 5, 10, 15, 20]
    c.most = 0
    assert c.check(kv)["lens"] == [1, 2, 3, 4]


def test_requests_that_do_not_exist_take_no_part(kv):
    ref = Case(random.Random(5), [-1, 5, -3], [4, 1, 0], 16, spare=3).check(kv)
    assert ref["full"] and ref["lens"] == [-1, 6, -3] and ref["slots"][:4] == [-1] * 4


def test_bad_page_ids(kv):
    c = Case(random.Random(6), [20, 40, 5], [2, -1, 1], 16, spare=3)
    c.tables[0][1] = c.n_pages                      # the page that the new tokens go to
    c.tables[1][1] = -1                             # dropped before: not given back
    c.tables[1][2] = -4                             # no page: left out and reported
    ref = c.check(kv)
    assert ref["bad"] and ref["slots"][:2] == [-1, -1] and ref["state"][1] == 4
    c = Case(random.Random(6), [16], [20], 16, spare=3)
    c.ring[c.head] = 99                             # a free page that is none
    ref = c.check(kv)
    assert ref["bad"] and ref["slots"][:16] == [-1] * 16 and min(ref["slots"][16:]) >= 0


def test_a_ring_that_would_hold_more_pages_than_there_are(kv):
    c = Case(random.Random(7), [64, 48], [-1, -1], 16, spare=5)
    c.count += 4                                    # four of the places behind the free ones are taken to be free as well
    ref = c.check(kv)
    assert ref["bad"] and ref["state"][1] == c.n_pages


@pytest.mark.parametrize("head,count", [(-1, 3), (12, 3), (0, -1), (0, 13), (1 << 30, 1 << 30)])
def test_a_ring_state_out_of_range(kv, head, count):
    c = Case(random.Random(8), [16, 17], [16, 3], 16, spare=9)
    assert c.n_pages == 12
    c.head, c.count = head, count
    ref = c.check(kv)
    assert ref["bad"] and ref["full"] and ref["lens"] == [16, 20]


def test_lengths_at_the_end_of_32_bits(kv):
    """Sums that pass 32 bits are refused, not wrapped: rows, tokens of a request, pages."""
    big = 2 ** 31 - 1
    ref = lib.plan([5, 0, 7], [big, big, 1], [[0, 1]] * 3, list(range(8)), 0, 0, 16, 4)
    assert ref["lens"] == [5, 0, 7]
    from paper_2605_22718_b200 import PagedKV
    c = PagedKV(kv, n_pages=8, page_tokens=16)
    lens, state = gpu([5, 0, big]), gpu([0, 8, 0, 0])
    tables = gpu([[0, 1]] * 3)
    slots, starts = c.page_plan(lens, gpu([big, big, big]), tables, gpu(list(range(8))), state, 4)
    assert lens.tolist() == [5, 0, big] and slots.tolist() == [-1] * 4 and starts.tolist() == [0, big, big, big]
    assert state.tolist() == [0, 8, 0, 0] and kv.poll_status()[1] == 8


@pytest.mark.parametrize("n_pages,steps", [(64, 200), (600, 120)])
def test_pages_go_round(kv, n_pages, steps):
    """Many steps on one ring: no page is ever held twice, and all come back."""
    from paper_2605_22718_b200 import PagedKV
    rng = random.Random(n_pages)
    page, n, width = 4, 24, 40
    c = PagedKV(kv, n_pages=n_pages, page_tokens=page)
    ring, state = c.free_pages()
    lens, tables = gpu([0] * n), gpu([[-1] * width] * n)
    h_lens, h_tables, h_ring, h_state = [0] * n, tables.tolist(), ring.tolist(), state.tolist()
    for _ in range(steps):
        new = [rng.choice([0, 1, 1, 7, -1]) if rng.random() < 0.98 else rng.randrange(60) for _ in range(n)]
        most = sum(max(0, v) for v in new)
        ref = lib.plan(h_lens, new, h_tables, h_ring, h_state[0], h_state[1], page, most)
        slots, _ = c.page_plan(lens, gpu(new), tables, ring, state, most)
        assert slots.tolist() == ref["slots"]
        h_lens, h_tables, h_ring, h_state = ref["lens"], ref["tables"], ref["ring"], ref["state"]
        held = [p for r in range(n) for p in h_tables[r][:-(-h_lens[r] // page)]]
        free = [h_ring[(h_state[0] + i) % n_pages] for i in range(h_state[1])]
        assert sorted(held + free) == list(range(n_pages))
    assert (lens.tolist(), tables.tolist(), ring.tolist(), state.tolist()) == (h_lens, h_tables, h_ring, h_state)
    c.page_plan(lens, gpu([-1] * n), tables, ring, state, 0)
    assert state.tolist()[1] == n_pages and lens.tolist() == [0] * n
    kv.poll_status()
