"""Plan, store and attention as a program uses them: step after step, on a stream of its own, and captured into a graph."""
import random

import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=2, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


def gpu(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Program:
    """Sessions that grow token by token, and what every layer's cache should hold."""

    def __init__(self, kv, type_, n=5, heads=8, kv_heads=4, d=128, page=8, n_pages=200, width=40, layers=2):
        from paper_2605_22718_b200 import PagedKV
        self.n, self.heads, self.kv_heads, self.d, self.type = n, heads, kv_heads, d, type_
        self.caches = [PagedKV.empty(kv, n_pages, page, kv_heads, d, lib.TYPES[type_]) for _ in range(layers)]
        self.ring, self.state = self.caches[0].free_pages()
        self.lens, self.tables = gpu([0] * n), gpu([[-1] * width] * n)
        self.history = [[[] for _ in range(n)] for _ in range(layers)]
        self.gen = torch.Generator(device="cuda").manual_seed(5)

    def rows(self, count):
        qkv = torch.randn((count, self.heads + 2 * self.kv_heads, self.d), generator=self.gen, device="cuda")
        return qkv.to(torch.bfloat16)

    def split(self, qkv):
        h, k = self.heads, self.kv_heads
        return qkv[:, :h], qkv[:, h:h + k], qkv[:, h + k:]

    def remember(self, layer, new, qkv):
        _, K, V = self.split(qkv)
        at = 0
        for r, m in enumerate(new):
            if m < 0:
                self.history[layer][r] = []
            for _ in range(max(0, m)):
                self.history[layer][r].append((K[at].clone(), V[at].clone()))
                at += 1

    def expect(self, layer, Q):
        """The formula over what was stored, as a cache of one page per session."""
        hist = self.history[layer]
        longest = max(1, max(len(h) for h in hist))
        K = torch.zeros((self.n, longest, self.kv_heads, self.d), dtype=torch.bfloat16, device="cuda")
        V = torch.zeros_like(K)
        for r, h in enumerate(hist):
            for t, (k, v) in enumerate(h):
                K[r, t], V[r, t] = k, v
        ke = ve = None
        if self.type == "e4m3":
            (kc, ke), (vc, ve) = lib.quantise(K), lib.quantise(V)
            K, V = (x.float().to(torch.float8_e4m3fn).cuda() for x in (kc, vc))
            ke, ve = ke.transpose(1, 2).contiguous().cuda(), ve.transpose(1, 2).contiguous().cuda()
        tables = torch.arange(self.n, dtype=torch.int32, device="cuda")[:, None]
        return lib.attend(Q, K, V, ke, ve, tables, [len(h) for h in hist])


@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
def test_sessions_that_come_grow_and_end(kv, type_):
    rng = random.Random(2)
    p = Program(kv, type_)
    side = torch.cuda.Stream()
    for step in range(24):
        new = [rng.choice([1, 1, 1, 0, 13, -1 if step > 3 else 1]) for _ in range(p.n)]
        most = sum(max(0, v) for v in new)
        dev_new = gpu(new)
        inputs = [p.rows(most) for _ in p.caches]
        Qs = [p.rows(p.n)[:, :p.heads] for _ in p.caches]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side) if step % 2 else torch.cuda.stream(torch.cuda.current_stream()):
            slots, _ = p.caches[0].page_plan(p.lens, dev_new, p.tables, p.ring, p.state, most)
            outs = []
            for c, qkv, Q in zip(p.caches, inputs, Qs):
                _, K, V = p.split(qkv)
                c.page_store(K, V, slots)
                lse = torch.empty((p.n, p.heads), device="cuda")
                outs.append((c.paged_attention(Q, p.tables, p.lens, lse_out=lse), lse))
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for layer, (O, lse) in enumerate(outs):
            p.remember(layer, new, inputs[layer])
            lib.assert_attends(O, lse, p.expect(layer, Qs[layer]))
        assert p.lens.tolist() == [len(h) for h in p.history[0]]
    assert kv.poll_status() == (0, 0)


@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
def test_a_captured_step_follows_the_lengths(kv, type_):
    """One token per session and replay; a padded row takes no part; another graph on the same scratch in between."""
    p = Program(kv, type_, n=4)
    prompt = [5, 0, 30, 0]
    qkv = [p.rows(35) for _ in p.caches]
    slots, _ = p.caches[0].page_plan(p.lens, gpu(prompt), p.tables, p.ring, p.state, 35)
    for layer, c in enumerate(p.caches):
        c.page_store(*p.split(qkv[layer])[1:], slots)
        p.remember(layer, prompt, qkv[layer])
    p.lens[3] = -1
    one = gpu([1, 1, 1, 0])
    static = [p.rows(3) for _ in p.caches]
    Qs = [p.rows(4)[:, :p.heads] for _ in p.caches]
    lses = [torch.full((4, p.heads), 7.0, device="cuda") for _ in p.caches]
    outs = [torch.full((4, p.heads, p.d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in p.caches]
    slots = torch.empty(4, dtype=torch.int32, device="cuda")
    starts = torch.empty(5, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()

    def step():
        p.caches[0].page_plan(p.lens, one, p.tables, p.ring, p.state, 4, slots_out=slots, starts_out=starts)
        for c, x, Q, O, lse in zip(p.caches, static, Qs, outs, lses):
            c.page_store(*p.split(x)[1:], slots)
            c.paged_attention(Q, p.tables, p.lens, O=O, lse_out=lse)

    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    spare = torch.empty_like(outs[0])
    with torch.cuda.graph(other):
        p.caches[1].paged_attention(Qs[1], p.tables, p.lens, O=spare)
    for i in range(20):
        for x in static:
            x.copy_(p.rows(3))
        graph.replay()
        if i % 3 == 0:
            other.replay()
        torch.cuda.synchronize()
        for layer in range(len(p.caches)):
            p.remember(layer, [1, 1, 1, 0], static[layer])
            ref = p.expect(layer, Qs[layer])
            lib.assert_attends(outs[layer][:3], lses[layer][:3], [x[:3] for x in ref])
            assert (outs[layer][3] == 9).all() and (lses[layer][3] == 7).all()
        assert p.lens.tolist() == [len(h) for h in p.history[0]][:3] + [-1] and slots[3] == -1
    del graph, other
    assert kv.poll_status() == (0, 0)


def test_two_calls_at_once_with_scratch_of_their_own(kv):
    from paper_2605_22718_b200 import PagedKV
    K, V, _, _ = lib.cache("bf16", 300, 16, 4, 128)
    c = PagedKV(kv, K, V)
    tables = torch.randperm(300).int().view(2, 150).cuda()
    lens = gpu([2400, 1777])
    Q = torch.randn((2, 16, 128), device="cuda").to(torch.bfloat16)
    want = c.paged_attention(Q, tables, lens)
    scratch = [torch.zeros_like(kv.paged_scratch) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                outs[i].append(c.paged_attention(Q, tables, lens, scratch=scratch[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for one in outs for o in one)


def test_a_context_that_is_not_bound_has_no_status_word(kv):
    """The C calls on an unbound context: the same results, nothing reported."""
    import ctypes as C
    from paper_2605_22718_b200 import PagedKV, WK_OK, load_library, wk_config
    L = load_library()
    h = C.c_void_p()
    assert L.wk_create(C.byref(wk_config(1, 1, 128, 8, 3, 4, 1, 1, 1, 0, 0.0, 0)), C.byref(h)) == WK_OK
    K, V, _, _ = lib.cache("bf16", 8, 16, 4, 128)
    c = PagedKV(kv, K, V)
    tables, lens = gpu([[3, 99, 1]]), gpu([40])
    Q = torch.randn((1, 8, 128), device="cuda").to(torch.bfloat16)
    want = c.paged_attention(Q, tables, lens)
    assert kv.poll_status()[1] == 1
    O, scratch = torch.empty_like(Q), torch.zeros(L.wk_paged_scratch_bytes(h), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert L.wk_paged_attention(h, c._desc_at, Q.data_ptr(), 0, 8 * 128, 1, 8, tables.data_ptr(), 3, 3, lens.data_ptr(), 0, 0, 0.0,
                                O.data_ptr(), None, scratch.data_ptr(), scratch.numel(), None) == WK_OK
    torch.cuda.synchronize()
    assert torch.equal(O, want) and kv.poll_status() == (0, 0)
    L.wk_destroy(h)


@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
def test_first_calls_inside_a_capture(type_):
    """A context's first plan, store and attention may be captured ones."""
    from paper_2605_22718_b200 import PagedKV, WorldKV
    fresh = WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)
    c = PagedKV.empty(fresh, 20, 16, 4, 128, lib.TYPES[type_])
    ring, state = c.free_pages()
    lens, tables = gpu([0, 0]), gpu([[-1] * 10] * 2)
    x = torch.randn((40, 4, 128), device="cuda").to(torch.bfloat16)
    Q = torch.randn((2, 12, 128), device="cuda").to(torch.bfloat16)
    new = gpu([33, 7])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slots, _ = c.page_plan(lens, new, tables, ring, state, 40)
        c.page_store(x, x, slots)
        O = c.paged_attention(Q, tables, lens)
    graph.replay()
    torch.cuda.synchronize()
    assert lens.tolist() == [33, 7] and state.tolist() == [4, 16, 0, 0]
    ref = lib.attend(Q, c.K, c.V, c.K_exp, c.V_exp, tables, [33, 7])
    lib.assert_attends(O, ref[1].float(), ref)
    del graph
    assert fresh.poll_status() == (0, 0)


def test_what_the_kernel_in_front_has_written_is_seen(kv):
    """Plans, stores and attentions one after the other without a pause, each needing what the one before has just written: the
    same results as with a wait after every call."""
    from paper_2605_22718_b200 import PagedKV
    n, page = 64, 4

    def run(wait):
        c = PagedKV.empty(kv, 64 * 40, page, 4, 64)
        ring, state = c.free_pages()
        lens, tables = gpu([0] * n), torch.full((n, 40), -1, dtype=torch.int32, device="cuda")
        g = torch.Generator(device="cuda").manual_seed(1)
        xs = [torch.randn((n * 3, 4, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(24)]
        Q = torch.randn((n, 8, 64), generator=g, device="cuda").to(torch.bfloat16)
        outs = []
        three = gpu([3] * n)
        for x in xs:
            slots, _ = c.page_plan(lens, three, tables, ring, state, 3 * n)
            if wait:
                torch.cuda.synchronize()
            c.page_store(x, x, slots)
            if wait:
                torch.cuda.synchronize()
            outs.append(c.paged_attention(Q, tables, lens))
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return outs

    want = run(True)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(run(False), want))
