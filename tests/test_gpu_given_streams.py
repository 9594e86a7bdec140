"""Calls that are given a stream: what they allocate belongs to that stream, not to the current one."""
import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=2, tokens_per_frame=8, n_keep=4, pool_slots=4, max_k=4)


def gpu(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def pages(kv):
    """A paged cache, and its three calls as functions of a stream that return what they allocate."""
    from paper_2605_22718_b200 import PagedKV
    K, V, _, _ = lib.cache("bf16", 80, 16, 4, 128)
    c = PagedKV(kv, K, V)
    tables, lens = torch.arange(80, dtype=torch.int32, device="cuda").view(2, 40), gpu([300, 17])
    Q = torch.randn((2, 16, 128), device="cuda").to(torch.bfloat16)
    ring, state = c.free_pages()
    few, many = [gpu(v) for v in ([0, 0], [3, 4], [[-1] * 4] * 2)], [gpu(v) for v in ([0] * 900, [0] * 900, [[-1] * 4] * 900)]
    torch.cuda.synchronize()
    return dict(
        slots=lambda s: c.page_plan(*few, ring, state, 1500, stream=s)[0],
        starts=lambda s: c.page_plan(*many, ring, state, 0, stream=s)[1],
        O=lambda s: c.paged_attention(Q, tables, lens, stream=s))


@pytest.mark.parametrize("what", ["slots", "starts", "O"])
def test_memory_of_a_result_stays_with_its_stream(kv, what):
    """A result that nobody holds is not handed out to the current stream, and one of the current stream's is not taken for a
    result on another: with either, two streams would use the same memory without waiting for one another."""
    call, side = pages(kv)[what], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x = call(side)
    at, shape = x.data_ptr(), (x.shape, x.dtype)
    del x
    mine = [torch.empty(shape[0], dtype=shape[1], device="cuda") for _ in range(4)]
    assert at not in [m.data_ptr() for m in mine]
    with torch.cuda.stream(side):
        assert torch.empty(shape[0], dtype=shape[1], device="cuda").data_ptr() == at          # it went back to its own stream
    theirs = [m.data_ptr() for m in mine]
    del mine
    assert call(side).data_ptr() not in theirs
    torch.cuda.synchronize()


@pytest.mark.parametrize("stream", [None, 0, "current", "default"])
def test_results_of_the_current_stream_are_as_before(kv, stream):
    s = {"current": torch.cuda.current_stream(), "default": torch.cuda.default_stream()}.get(stream, stream)
    for call in pages(kv).values():
        x = call(s)
        at, shape, dtype = x.data_ptr(), x.shape, x.dtype
        del x
        assert torch.empty(shape, dtype=dtype, device="cuda").data_ptr() == at
    torch.cuda.synchronize()


def chunks(score_mode=0):
    """The chunk pool's calls that allocate, as functions of a stream."""
    from paper_2605_22718_b200 import WorldKV
    T, H, F = 8, 2, 3
    kv = WorldKV(n_layers=1, n_heads=H, tokens_per_frame=T, n_keep=4, pool_slots=4, max_k=700, max_lq=64, score_mode=score_mode)
    g = torch.Generator(device="cuda").manual_seed(4)
    K, V = (torch.randn((1, F * T, H * 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    poses = torch.randn((5000, 8), generator=g, device="cuda")
    Q = torch.randn((40, H, 128), generator=g, device="cuda").to(torch.bfloat16)
    pose = [0.0] * 8
    slot, _, _ = kv.pool_compress_append(0, 1, K, V, pose)
    seg = (K[0].view(-1, H, 128), V[0].view(-1, H, 128))
    slots, scratch = gpu([slot]), torch.empty(kv.lib.wk_retrieve_scan_scratch_bytes(), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    return kv, dict(
        compress_chunk=lambda s: kv.compress_chunk(K, stream=s),
        compress_append=lambda s: kv.pool_compress_append(0, 1, K, V, pose, evict_oldest_if_full=True, stream=s)[2],
        retrieve=lambda s: kv.retrieve(pose, 1, stream=s)[0],
        retrieve_scan=lambda s: kv.retrieve_scan(poses, pose, 20, scratch=scratch, stream=s),
        retrieve_query=lambda s: kv.retrieve_query(0, Q, 1, stream=s)[0],
        memory_attention=lambda s: kv.memory_attention(0, Q, [seg], slots, 1, stream=s))


@pytest.mark.parametrize("what", ["compress_chunk", "compress_append", "retrieve", "retrieve_scan", "retrieve_query", "memory_attention"])
def test_memory_of_the_chunk_pools_results_stays_with_its_stream(what):
    kv, calls = chunks()
    call, side = calls[what], torch.cuda.Stream()
    x = call(side)
    at, shape, dtype = x.data_ptr(), x.shape, x.dtype
    del x
    mine = [torch.empty(shape, dtype=dtype, device="cuda") for _ in range(4)]
    assert at not in [m.data_ptr() for m in mine]
    with torch.cuda.stream(side):
        assert torch.empty(shape, dtype=dtype, device="cuda").data_ptr() == at
    theirs = [m.data_ptr() for m in mine]
    del mine
    assert call(side).data_ptr() not in theirs
    torch.cuda.synchronize()
    for s in (None, 0, torch.cuda.current_stream()):
        x = call(s)
        at = x.data_ptr()
        del x
        assert torch.empty(shape, dtype=dtype, device="cuda").data_ptr() == at
    torch.cuda.synchronize()


def test_a_stream_object_of_another_kind():
    """All that is asked of a stream is its handle."""
    class Stream:
        def __init__(self, s):
            self.cuda_stream = s.cuda_stream
    kv, calls = chunks()
    want = calls["memory_attention"](None).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = calls["memory_attention"](Stream(side))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    got = pages(kv)["O"](Stream(side))
    torch.cuda.synchronize()
    assert torch.isfinite(got).all()


def test_steps_on_a_given_stream(kv):
    """Plan, store and attention on a stream of their own while the current one keeps allocating and overwriting blocks of the same
    sizes: the same results as one call after the other."""
    from paper_2605_22718_b200 import PagedKV

    def run(s):
        c = PagedKV.empty(kv, 400, 8, 4, 128)
        ring, state = c.free_pages()
        lens, tables = gpu([0] * 40), torch.full((40, 10), -1, dtype=torch.int32, device="cuda")
        g = torch.Generator(device="cuda").manual_seed(2)
        rows = [torch.randn((40 * 3, 4, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(20)]
        Q = torch.randn((40, 8, 128), generator=g, device="cuda").to(torch.bfloat16)
        new, outs = gpu([3] * 40), []
        torch.cuda.synchronize()
        for x in rows:
            slots, _ = c.page_plan(lens, new, tables, ring, state, 120, stream=s)
            c.page_store(x, x, slots, stream=s)
            outs.append(c.paged_attention(Q, tables, lens, stream=s))
            del slots
            for _ in range(3):
                torch.full((120,), 7, dtype=torch.int32, device="cuda")
                torch.full((40, 8, 128), 3.0, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        return outs

    want = run(None)
    assert all(torch.equal(a, b) for a, b in zip(run(torch.cuda.Stream()), want))
    assert kv.poll_status() == (0, 0)


def test_a_given_stream_inside_a_capture(kv):
    calls = pages(kv)
    want = calls["O"](None).clone()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        O = calls["O"](s)
    O.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, want)
    del graph
