"""What the token-level cache's calls refuse of CUDA tensors: one defect at a time, told by its message and status, nothing written."""
import pytest
import torch

import paged_testlib as lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2605_22718_b200 import WorldKV
    return WorldKV(n_layers=1, n_heads=1, tokens_per_frame=8, n_keep=4, pool_slots=1, max_k=1)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


def refused(call, status, says):
    from paper_2605_22718_b200 import WkError
    with pytest.raises(WkError) as e:
        call()
    assert e.value.status == status and says in str(e.value), (e.value.status, str(e.value))


ALIKE = "K and V of one shape, type and layout"


@pytest.mark.parametrize("what,defect", [
    (ALIKE, dict(V=lambda K, V: None)), (ALIKE, dict(V=lambda K, V: V[:3])), (ALIKE, dict(V=lambda K, V: V[:, :15])),
    (ALIKE, dict(V=lambda K, V: V[:, :, :7])), (ALIKE, dict(V=lambda K, V: V[..., :64])), (ALIKE, dict(V=lambda K, V: V.half())),
    (ALIKE, dict(V=lambda K, V: V.transpose(1, 2).contiguous().transpose(1, 2))),        # the same shape, other strides
    (ALIKE, dict(V=lambda K, V: torch.cat([V, V], 3)[..., :128])),
    (ALIKE, dict(K=lambda K, V: K.float(), V=lambda K, V: V.float())), (ALIKE, dict(K=lambda K, V: K[0], V=lambda K, V: V[0])),
    (ALIKE, dict(K=lambda K, V: K.transpose(2, 3), V=lambda K, V: V.transpose(2, 3))),   # the last axis in steps
    ("on the context's device", dict(V=lambda K, V: V.cpu())), ("on the context's device", dict(K=lambda K, V: K.cpu())),
    ("exponents belong", dict(ke=lambda K, V: torch.zeros((4, 8, 16), dtype=torch.uint8, device="cuda"))),
    ("exponents belong", dict(ve=lambda K, V: torch.zeros((4, 8, 16), dtype=torch.uint8, device="cuda"))),
])
def test_caches_of_16_bits(kv, what, defect):
    from paper_2605_22718_b200 import PagedKV, WK_ERR_ARG
    K, V = torch.zeros((4, 16, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 16, 8, 128), dtype=torch.bfloat16, device="cuda")
    PagedKV(kv, K, V)
    args = {name: defect[name](K, V) if name in defect else at for name, at in (("K", K), ("V", V), ("ke", None), ("ve", None))}
    refused(lambda: PagedKV(kv, *args.values()), WK_ERR_ARG, what)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("defect", [
    lambda e: None, lambda e: e[:2], lambda e: e[:, :4], lambda e: e[:, :, :8], lambda e: e.transpose(1, 2), lambda e: e.int(), lambda e: e.view(torch.int8),
    lambda e: torch.cat([e, e], 2)[:, :, :16], lambda e: e.reshape(-1), lambda e: e.transpose(1, 2).contiguous().transpose(1, 2)])
def test_exponents_of_8_bits(kv, which, defect):
    from paper_2605_22718_b200 import PagedKV, WK_ERR_ARG
    K, V, *exps = lib.cache("e4m3", 3, 16, 5, 128)
    PagedKV(kv, K, V, *exps)
    exps[which] = defect(exps[which])
    refused(lambda: PagedKV(kv, K, V, *exps), WK_ERR_ARG, "K_exp and V_exp")


def test_exponents_on_the_host(kv):
    from paper_2605_22718_b200 import PagedKV, WK_ERR_ARG
    K, V, ke, ve = lib.cache("e4m3", 3, 16, 5, 128)
    refused(lambda: PagedKV(kv, K, V, ke.cpu(), ve), WK_ERR_ARG, "on the context's device")
    refused(lambda: PagedKV(kv, K, V, ke, ve.cpu()), WK_ERR_ARG, "on the context's device")


PLAN = dict(lens=(3,), new_tokens=(3,), tables=(3, 4), ring=(8,), state=(4,), lens_out=(3,), state_out=(4,), slots_out=(6,), starts_out=(4,))
SAYS = dict(lens="lens", new_tokens="new_tokens", tables="tables", ring="ring", state="state", lens_out="lens_out", state_out="state_out",
            slots_out="slots_out", starts_out="starts_out")


@pytest.mark.parametrize("name", list(PLAN))
@pytest.mark.parametrize("defect", ["long", "host", "short", "steps", "nothing"])
def test_plans(kv, name, defect):
    """Each tensor of a plan in turn: another type, on the host, an element too few, not contiguous, none at all."""
    from paper_2605_22718_b200 import PagedKV, WK_ERR_ARG, WkError
    c = PagedKV(kv, n_pages=8, page_tokens=16)
    a = {k: i32(*s) for k, s in PLAN.items()}
    c.page_plan(max_tokens=6, **a)
    x = a[name]
    if name == "lens" and defect in ("short", "nothing"):
        return                                      # n_req is its size: fewer is a plan of fewer; none is no call
    if defect == "nothing":
        if name in ("lens_out", "state_out", "slots_out", "starts_out"):
            return                                  # allocated, or in place
        a[name] = None
    else:
        a[name] = {"long": lambda: x.long(), "host": lambda: x.cpu(), "short": lambda: x[:-1].contiguous(),
                   "steps": lambda: torch.cat([x, x], -1)[..., ::2]}[defect]()
    torch.cuda.synchronize()
    before = {k: v.clone() for k, v in a.items() if v is not None}
    refused(lambda: c.page_plan(max_tokens=6, **a), WK_ERR_ARG, SAYS[name])
    assert all(torch.equal(a[k], v) for k, v in before.items())
    for most in (-1, 2 ** 31):
        with pytest.raises(WkError):
            c.page_plan(i32(3), i32(3), i32(3, 4), i32(8), i32(4), most)


@pytest.mark.parametrize("says,defect", [
    ("K_new, V_new", dict(K=lambda x: x.float())), ("K_new, V_new", dict(V=lambda x: x.half())), ("K_new, V_new", dict(V=lambda x: x[:3])),
    ("K_new, V_new", dict(K=lambda x: x.cpu(), V=lambda x: x.cpu())), ("K_new, V_new", dict(K=lambda x: x[:, :7], V=lambda x: x[:, :7])),
    ("K_new, V_new", dict(K=lambda x: x[..., :64], V=lambda x: x[..., :64])), ("K_new, V_new", dict(K=lambda x: x.view(4, -1), V=lambda x: x.view(4, -1))),
    ("K_new, V_new", dict(V=lambda x: torch.cat([x, x], 1)[:, :8])),                                   # another row stride than K's
    ("K_new, V_new", dict(K=lambda x: x.transpose(1, 2).contiguous().transpose(1, 2), V=lambda x: x.transpose(1, 2).contiguous().transpose(1, 2))),
    ("K_new", dict(K=lambda x: None)), ("V_new", dict(V=lambda x: None)),
    ("slots", dict(slots=lambda x: x.long())), ("slots", dict(slots=lambda x: x[:3])), ("slots", dict(slots=lambda x: x.cpu())),
    ("slots", dict(slots=lambda x: torch.cat([x, x])[::2])), ("slots", dict(slots=lambda x: None)),
])
def test_stores(kv, says, defect):
    from paper_2605_22718_b200 import PagedKV, WK_ERR_ARG
    K, V, _, _ = lib.cache("bf16", 2, 16, 8, 128)
    old = K.clone(), V.clone()
    x = torch.ones((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    a = dict(K=x, V=x.clone(), slots=i32(4))
    a.update({k: f(a[k]) for k, f in defect.items()})
    refused(lambda: PagedKV(kv, K, V).page_store(a["K"], a["V"], a["slots"]), WK_ERR_ARG, says)
    torch.cuda.synchronize()
    assert torch.equal(K, old[0]) and torch.equal(V, old[1])


def test_types_that_do_not_go_together(kv):
    """What the library itself refuses has its status."""
    from paper_2605_22718_b200 import PagedKV, WK_ERR_ARG, WK_ERR_SHAPE
    x = torch.ones((4, 8, 128), dtype=torch.float16, device="cuda")
    K, V, _, _ = lib.cache("bf16", 2, 16, 8, 128)
    refused(lambda: PagedKV(kv, K, V).page_store(x, x, i32(4)), WK_ERR_ARG, "wk_page_store")
    K8, V8, *exps = lib.cache("e4m3", 2, 16, 8, 128)
    codes = x.to(torch.float8_e4m3fn)
    refused(lambda: PagedKV(kv, K8, V8, *exps).page_store(codes, codes, i32(4)), WK_ERR_ARG, "wk_page_store")
    refused(lambda: PagedKV(kv, K8, V8, *exps).paged_attention(codes, i32(4, 2), i32(4)), WK_ERR_ARG, "wk_paged_attention")
    q = torch.ones((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    c = PagedKV(kv, K, V)
    for args, kw, status, says in [
            ((q[:, :6].contiguous(), i32(4, 2), i32(4)), {}, WK_ERR_SHAPE, "wk_paged_attention"),      # 6 heads over 8
            ((q.half(), i32(4, 2), i32(4)), {}, WK_ERR_ARG, "wk_paged_attention"), ((q.float(), i32(4, 2), i32(4)), {}, WK_ERR_ARG, "Q [n_req"),
            ((q[..., :64], i32(4, 2), i32(4)), {}, WK_ERR_ARG, "Q [n_req"), ((q.cpu(), i32(4, 2), i32(4)), {}, WK_ERR_ARG, "Q [n_req"),
            ((q.transpose(1, 2).contiguous().transpose(1, 2), i32(4, 2), i32(4)), {}, WK_ERR_ARG, "Q [n_req"),
            ((q, i32(4, 2).long(), i32(4)), {}, WK_ERR_ARG, "tables"), ((q, i32(3, 2), i32(4)), {}, WK_ERR_ARG, "tables"),
            ((q, i32(4, 0), i32(4)), {}, WK_ERR_ARG, "wk_paged_attention"), ((q, i32(2, 4).t(), i32(4)), {}, WK_ERR_ARG, "tables"),
            ((q, i32(4, 2), i32(4).long()), {}, WK_ERR_ARG, "lens"), ((q, i32(4, 2), i32(3)), {}, WK_ERR_ARG, "lens"),
            ((q, i32(4, 2), i32(4)), dict(O=q.float()), WK_ERR_ARG, "O like Q"), ((q, i32(4, 2), i32(4)), dict(O=q[:3]), WK_ERR_ARG, "O like Q"),
            ((q, i32(4, 2), i32(4)), dict(O=torch.cat([q, q], 1)[:, :8]), WK_ERR_ARG, "O like Q"),
            ((q, i32(4, 2), i32(4)), dict(lse_out=q), WK_ERR_ARG, "lse_out"), ((q, i32(4, 2), i32(4)), dict(lse_out=torch.zeros((8, 4), device="cuda").t()), WK_ERR_ARG, "lse_out"),
            ((q, i32(4, 2), i32(4)), dict(window=-1), WK_ERR_ARG, "wk_paged_attention"), ((q, i32(4, 2), i32(4)), dict(sink=-1), WK_ERR_ARG, "wk_paged_attention"),
            ((q, i32(4, 2), i32(4)), dict(window=2 ** 31), WK_ERR_ARG, "window"), ((q, i32(4, 2), i32(4)), dict(softmax_scale=-0.5), WK_ERR_ARG, "wk_paged_attention"),
            ((q, i32(4, 2), i32(4)), dict(scratch=torch.zeros(256, dtype=torch.uint8, device="cuda")), WK_ERR_SHAPE, "wk_paged_attention"),
            ((q, i32(4, 2), i32(4)), dict(scratch=torch.zeros_like(kv.paged_scratch).cpu()), WK_ERR_ARG, "scratch"),
            ((q, i32(4, 2), i32(4)), dict(scratch=torch.zeros(kv.paged_scratch.numel() + 16, dtype=torch.uint8, device="cuda")[16:]), WK_ERR_ARG, "wk_paged_attention")]:
        refused(lambda: c.paged_attention(*args, **kw), status, says)
    assert kv.poll_status() == (0, 0)
