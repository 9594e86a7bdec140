"""What the token-level cache's binding refuses before anything reaches the library, each defect told by its message.  No GPU needed."""
import pytest
import torch

from paper_2605_22718_b200 import binding

ARG = binding.WK_ERR_ARG


class Context:
    """A context that is none: enough for what is refused before a call."""
    lib, device, ctx = None, torch.device("cuda", 0), None


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("name,args,kw", [
    ("page_store", (torch.zeros((4, 8, 128)), torch.zeros((4, 8, 128)), i32(4)), {}),
    ("paged_attention", (torch.zeros((4, 8, 128)), i32(4, 2), i32(4)), {}),
    ("paged_attention", (torch.zeros((4, 8, 128)), i32(4, 2), i32(4)), dict(scratch=torch.zeros(512, dtype=torch.uint8)))])
def test_a_cache_that_only_plans_neither_stores_nor_attends(name, args, kw):
    only_plans = binding.PagedKV(Context, n_pages=3, page_tokens=16)
    with pytest.raises(binding.WkError) as e:
        getattr(only_plans, name)(*args, **kw)
    assert e.value.status == ARG and "only plans" in str(e.value)


@pytest.mark.parametrize("K,V", [
    (0, lambda x: None), (0, lambda x: x[:3]), (0, lambda x: x.half()), (0, lambda x: x[..., :64]),
    (0, lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)), (lambda x: x.float(), lambda x: x.float()),
    (lambda x: x.transpose(2, 3), lambda x: x.transpose(2, 3)), (lambda x: x[0], lambda x: x[0])])
def test_keys_and_values_that_are_not_alike(K, V):
    """Refused for what they are, before it matters where they are."""
    x = torch.zeros((4, 16, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(binding.WkError) as e:
        binding.PagedKV(Context, K(x) if K else x, V(x))
    assert e.value.status == ARG and "of one shape, type and layout" in str(e.value)


def test_a_cache_of_nothing():
    for kw in (dict(), dict(n_pages=3), dict(page_tokens=16)):
        with pytest.raises(binding.WkError) as e:
            binding.PagedKV(Context, **kw)
        assert e.value.status == ARG and "n_pages and page_tokens" in str(e.value)
