"""Argument checks of the token-level cache's entry points (csrc/wk_paged_api.cu), built against stand-ins for the CUDA runtime and the
launchers: what is refused, with which status, before anything is launched.  No GPU needed."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2605_22718_b200 import binding
from paper_2605_22718_b200.build import CSRC, ROOT, _nvcc

OK, ARG, SHAPE = binding.WK_OK, binding.WK_ERR_ARG, binding.WK_ERR_SHAPE
P = 0x10000            # an address that is aligned and never looked at
I32MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    out = str(tmp_path_factory.mktemp("host") / "libwk_paged_host.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-I", cuda, "-I", CSRC, "-x", "c++",
                    os.path.join(CSRC, "wk_api.cu"), os.path.join(CSRC, "wk_paged_api.cu"),
                    os.path.join(ROOT, "tests", "host", "fake_device.cc"), os.path.join(ROOT, "tests", "host", "fake_pages.cc"),
                    "-o", out], check=True)
    lib = C.CDLL(out)
    real = binding.load_library()
    for name in ("wk_page_plan", "wk_page_store", "wk_paged_attention", "wk_paged_scratch_bytes", "wk_create"):
        getattr(lib, name).argtypes, getattr(lib, name).restype = getattr(real, name).argtypes, getattr(real, name).restype
    return lib


@pytest.fixture
def ctx(lib):
    cfg = binding.wk_config(1, 1, 128, 4, 3, 2, 1, 1, 1, 0, 0.0, 0)
    h = C.c_void_p()
    assert lib.wk_create(C.byref(cfg), C.byref(h)) == OK
    C.c_int.in_dll(lib, "launched").value = 0
    yield h
    lib.wk_destroy(h)


def launched(lib):
    return C.c_int.in_dll(lib, "launched").value


def desc(**kw):
    d = dict(K=P, V=P, K_exp=None, V_exp=None, page_stride=16 * 8 * 128, token_stride=8 * 128, head_stride=128, n_pages=10,
             page_tokens=16, n_kv_heads=8, head_dim=128, type=binding.WK_BF16, reserved=0)
    d.update(kw)
    return binding.wk_paged_kv(*[d[name] for name, _ in binding.wk_paged_kv._fields_])


E4M3 = dict(type=binding.WK_E4M3, K_exp=P, V_exp=P)
BAD_CACHES = [
    (dict(K=None), ARG), (dict(V=None), ARG), (dict(K=P + 8), ARG), (dict(V=P + 2), ARG), (dict(type=3), ARG), (dict(type=-1), ARG),
    (dict(head_dim=96), ARG), (dict(head_dim=0), ARG), (dict(n_pages=0), ARG), (dict(page_tokens=0), ARG), (dict(n_kv_heads=0), ARG),
    (dict(reserved=1), ARG), (dict(K_exp=P), ARG), (dict(type=binding.WK_E4M3), ARG), (dict(E4M3, V_exp=None), ARG), (dict(E4M3, K_exp=P + 2), ARG), (dict(E4M3, V_exp=P + 1), ARG),
    (dict(token_stride=8 * 128 + 4), ARG), (dict(head_stride=127), ARG), (dict(page_stride=-16 * 8 * 128), ARG),
    (dict(E4M3, token_stride=8 * 128 + 8), ARG),                       # 8 bytes
    (dict(head_stride=120), ARG), (dict(token_stride=7 * 128), ARG), (dict(page_stride=15 * 8 * 128), ARG),   # rows overlap
    (dict(page_stride=0), ARG), (dict(token_stride=128), ARG),
    (dict(n_pages=1 << 27), SHAPE),                                    # 2^31 slots
    (dict(E4M3, n_pages=1 << 25, n_kv_heads=8), SHAPE),                # 2^32 exponents
]
GOOD_CACHES = [
    dict(), E4M3, dict(type=binding.WK_F16, head_dim=64), dict(n_pages=1, page_stride=3), dict(page_tokens=1, token_stride=0),
    dict(n_kv_heads=1, head_stride=5), dict(head_stride=16 * 128, token_stride=128),                # heads outside tokens
    dict(page_stride=2 * 16 * 8 * 128), dict(token_stride=8 * 160, head_stride=160, page_stride=16 * 8 * 160),
]


def store(lib, ctx, cache, src=binding.WK_BF16, n=4, stride=8 * 128, K=P, V=P, slots=P):
    return lib.wk_page_store(ctx, C.addressof(cache) if cache else None, K, V, src, n, stride, slots, None)


def attend(lib, ctx, cache, Q=P, q_type=binding.WK_BF16, q_stride=16 * 128, n=4, heads=16, tables=P, max_pages=8,
           table_stride=8, lens=P, window=0, sink=0, scale=0.0, O=P, lse=None, scratch=P, scratch_bytes=512):
    return lib.wk_paged_attention(ctx, C.addressof(cache) if cache else None, Q, q_type, q_stride, n, heads, tables, max_pages,
                                  table_stride, lens, window, sink, scale, O, lse, scratch, scratch_bytes, None)


def plan(lib, ctx, n_pages=10, page=16, n=4, lens=P, new=P, lens_out=P, tables=P, max_pages=8, stride=8, ring=P, state=P,
         state_out=P, most=100, slots=P, starts=P):
    return lib.wk_page_plan(ctx, n_pages, page, n, lens, new, lens_out, tables, max_pages, stride, ring, state, state_out, most,
                            slots, starts, None)


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_caches_that_are_refused(lib, ctx, kw, status):
    src = binding.WK_BF16
    assert store(lib, ctx, desc(**kw), src) == status
    assert attend(lib, ctx, desc(**kw)) == status
    assert launched(lib) == 0


@pytest.mark.parametrize("kw", GOOD_CACHES)
def test_caches_that_are_accepted(lib, ctx, kw):
    c = desc(**kw)
    src = c.type if c.type != binding.WK_E4M3 else binding.WK_F16
    assert store(lib, ctx, c, src) == OK
    assert attend(lib, ctx, c, q_type=src) == OK
    assert launched(lib) == 2


@pytest.mark.parametrize("kw,status", [
    (dict(cache=None), ARG), (dict(src=binding.WK_F16), ARG), (dict(src=binding.WK_E4M3), ARG), (dict(n=-1), ARG),
    (dict(K=None), ARG), (dict(V=None), ARG), (dict(slots=None), ARG), (dict(K=P + 8), ARG), (dict(V=P + 4), ARG),
    (dict(stride=8 * 128 + 4), ARG), (dict(stride=7 * 128), ARG), (dict(stride=-8 * 128), ARG),
    (dict(cache=desc(**E4M3), src=binding.WK_E4M3), ARG)])
def test_stores_that_are_refused(lib, ctx, kw, status):
    kw = dict(dict(cache=desc()), **kw)
    assert store(lib, ctx, **kw) == status and launched(lib) == 0


def test_stores_that_are_accepted(lib, ctx):
    assert store(lib, ctx, desc(), n=0, K=None, V=None, slots=None) == OK and launched(lib) == 0     # nothing to do
    assert store(lib, ctx, desc(), n=1, stride=0) == OK
    assert store(lib, ctx, desc(), stride=24 * 128) == OK                                            # a slice of wider rows
    assert launched(lib) == 2
    assert store(lib, None, desc()) == ARG


@pytest.mark.parametrize("kw,status", [
    (dict(cache=None), ARG), (dict(Q=None), ARG), (dict(O=None), ARG), (dict(tables=None), ARG), (dict(lens=None), ARG),
    (dict(scratch=None), ARG), (dict(q_type=binding.WK_F16), ARG), (dict(q_type=binding.WK_E4M3), ARG), (dict(q_type=7), ARG),
    (dict(n=0), ARG), (dict(heads=0), ARG), (dict(max_pages=0), ARG), (dict(window=-1), ARG), (dict(sink=-1), ARG),
    (dict(scale=-1.0), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(Q=P + 8), ARG),
    (dict(O=P + 8), ARG), (dict(scratch=P + 16), ARG), (dict(q_stride=16 * 128 + 4), ARG), (dict(q_stride=15 * 128), ARG),
    (dict(table_stride=7), ARG), (dict(heads=12), SHAPE), (dict(scratch_bytes=511), SHAPE),
    (dict(cache=desc(page_stride=1 << 32, n_pages=100)), SHAPE),                                     # places beyond 32 bits of 16 bytes
    (dict(cache=desc(**E4M3), q_type=binding.WK_E4M3), ARG)])
def test_attentions_that_are_refused(lib, ctx, kw, status):
    kw = dict(dict(cache=desc()), **kw)
    assert attend(lib, ctx, **kw) == status and launched(lib) == 0


def test_attentions_that_are_accepted(lib, ctx):
    value = lambda name, t=C.c_int: t.in_dll(lib, name).value  # noqa: E731
    assert attend(lib, ctx, desc(), n=1, q_stride=0, table_stride=0) == OK
    assert abs(value("last_scale", C.c_float) - 128 ** -0.5) < 1e-8
    assert attend(lib, ctx, desc(), scale=0.25, window=100, sink=7) == OK
    assert value("last_scale", C.c_float) == 0.25 and (value("last_window"), value("last_sink")) == (100, 7)
    assert attend(lib, ctx, desc(), window=I32MAX, sink=I32MAX) == OK and (value("last_window"), value("last_sink")) == (0, 0)
    assert attend(lib, ctx, desc(), window=0, sink=5) == OK and (value("last_window"), value("last_sink")) == (0, 0)
    assert attend(lib, ctx, desc(), max_pages=I32MAX, table_stride=I32MAX) == OK
    assert value("last_max_pages") == I32MAX // 16                   # positions stay below 2^31
    assert attend(lib, None, desc()) == ARG
    assert lib.wk_paged_scratch_bytes(None) == 0 and lib.wk_paged_scratch_bytes(ctx) == 512


@pytest.mark.parametrize("kw,status", [
    *[({name: None}, ARG) for name in ("lens", "new", "lens_out", "tables", "ring", "state", "state_out", "slots", "starts")],
    (dict(n_pages=0), ARG), (dict(page=0), ARG), (dict(n=0), ARG), (dict(max_pages=0), ARG), (dict(most=-1), ARG),
    (dict(stride=7), ARG), (dict(n=4097), SHAPE), (dict(max_pages=1 << 30, stride=1 << 30), SHAPE), (dict(n_pages=1 << 27), SHAPE)])
def test_plans_that_are_refused(lib, ctx, kw, status):
    assert plan(lib, ctx, **kw) == status and launched(lib) == 0


def test_plans_that_are_accepted(lib, ctx):
    assert plan(lib, ctx) == OK and plan(lib, ctx, most=0, slots=None) == OK and plan(lib, ctx, n=4096) == OK
    assert plan(lib, ctx, n=1, stride=0) == OK and launched(lib) == 4
    assert plan(lib, None) == ARG


def test_tensors_that_the_binding_refuses():
    """What a C call cannot see: types, shapes, layouts and places of tensors."""
    class Context:
        lib, device, ctx = None, torch.device("cuda", 0), None
    cpu = torch.zeros((4, 16, 8, 128), dtype=torch.bfloat16)
    for bad in (dict(K=cpu, V=cpu), dict(K=cpu, V=None), dict(K=cpu, V=cpu[:3]), dict(K=cpu.float(), V=cpu.float()),
                dict(K=cpu.transpose(2, 3), V=cpu.transpose(2, 3)), dict(K=cpu, V=cpu.half()), dict(), dict(n_pages=3)):
        with pytest.raises(binding.WkError) as e:
            binding.PagedKV(Context, **bad)
        assert e.value.status == ARG
    only_plans = binding.PagedKV(Context, n_pages=3, page_tokens=16)
    with pytest.raises(binding.WkError):
        only_plans.page_plan(*[torch.zeros(4, dtype=torch.int32)] * 2, torch.zeros((4, 2), dtype=torch.int32),
                             torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), 0,
                             slots_out=torch.zeros(0, dtype=torch.int32), starts_out=torch.zeros(5, dtype=torch.int32))
