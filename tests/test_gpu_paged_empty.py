"""The token-level cache's calls on a batch without requests: nothing to do, on any stream, captured too."""
import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cache():
    from paper_2605_22718_b200 import PagedKV, WorldKV
    kv = WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)
    K, V, _, _ = lib.cache("bf16", 8, 16, 4, 128)
    return PagedKV(kv, K, V)


def nothing(width=5):
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    return none, none.clone(), torch.empty((0, width), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("most", [0, 1, 700])
@pytest.mark.parametrize("given", [False, True])
def test_a_plan_of_no_requests(cache, most, given):
    ring, state = cache.free_pages()
    state[0] = 3
    before = ring.clone(), state.clone()
    s = torch.cuda.Stream() if given else None
    torch.cuda.synchronize()
    slots, starts = cache.page_plan(*nothing(), ring, state, most, stream=s)
    torch.cuda.synchronize()
    assert slots.tolist() == [-1] * most and starts.tolist() == [0]
    assert torch.equal(ring, before[0]) and torch.equal(state, before[1])
    out, slots, starts = torch.full((4,), 9, dtype=torch.int32, device="cuda"), *(torch.full((800,), 9, dtype=torch.int32, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    got = cache.page_plan(*nothing(), ring, state, most, lens_out=nothing()[0], state_out=out, slots_out=slots, starts_out=starts, stream=s)
    torch.cuda.synchronize()
    assert got[0] is slots and got[1] is starts
    assert slots.tolist() == [-1] * most + [9] * (800 - most) and starts.tolist() == [0] + [9] * 799 and torch.equal(out, state)
    assert cache.kv.poll_status() == (0, 0)


def test_a_step_of_no_requests(cache):
    ring, state = cache.free_pages()
    lens, new, tables = nothing()
    x, Q = (torch.empty((0, h, 128), dtype=torch.bfloat16, device="cuda") for h in (4, 8))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slots, starts = cache.page_plan(lens, new, tables, ring, state, 3)
        cache.page_store(x, x, slots)
        O = cache.paged_attention(Q, tables, lens)
    graph.replay()
    torch.cuda.synchronize()
    assert O.shape == (0, 8, 128) and slots.tolist() == [-1] * 3 and starts.tolist() == [0]
    del graph


def test_what_is_refused_all_the_same(cache):
    from paper_2605_22718_b200 import WkError, WK_ERR_ARG
    ring, state = cache.free_pages()
    for args in ((*nothing(), ring[:3], state, 1), (*nothing(), ring, state, -1), (*nothing(), ring, state[:3], 1)):
        with pytest.raises(WkError) as e:
            cache.page_plan(*args)
        assert e.value.status == WK_ERR_ARG
