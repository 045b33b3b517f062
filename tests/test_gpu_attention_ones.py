"""The stride of a dimension of one has no meaning: results do not depend on it and no call is refused for it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2601_07048_amd import jx  # noqa: E402
from test_gpu_attention import BF, Paged, found_case, i32, normal  # noqa: E402


def odd(x):
    """x with a stride of 13 in every dimension of one but the last."""
    return x.as_strided(x.shape, [13 if n == 1 and i + 1 < x.dim() else s for i, (n, s) in enumerate(zip(x.shape, x.stride()))], x.storage_offset())


@pytest.mark.parametrize("heads,kv,page,length", [(4, 1, 16, 100), (1, 1, 1, 20), (3, 1, 64, 64), (1, 1, 16, 16)])
def test_paged_attention(heads, kv, page, length):
    p = Paged(BF, heads, kv, 64, page, [length], [1], seed=1, spare=0)
    want = p.run()
    p.q, p.k = odd(p.q), odd(p.k)  # the values' strides stay
    got = p.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    p.v = odd(p.v)
    got = p.run()
    assert torch.equal(got[0], want[0])


def test_one_key_head_in_caches_of_two_orders():
    p = Paged(BF, 4, 1, 64, 16, [100], [5], seed=1)
    want = p.run()
    p.k = torch.empty((p.k.shape[0], 1, 16, 64), dtype=BF, device="cuda").transpose(1, 2).copy_(p.k)
    assert p.k.stride() != p.v.stride()
    assert torch.equal(p.run()[0], want[0])


def test_found_rows():
    q, keys, values, ids = found_case(BF, 1, 1, 1, 64, 5, 1, seed=2)
    want = jx.found_attention(q, keys, values, ids, 0.1)
    got = jx.found_attention(odd(q), odd(keys), values, ids, 0.1)
    assert torch.equal(got[0], want[0])


def test_norm_rotation_and_store():
    q, k, v = (normal((1, 1, 64), BF, i) for i in range(3))
    caches = [torch.zeros((1, 1, 1, 64), dtype=BF, device="cuda") for _ in range(4)]
    pos, slot = i32([0]), torch.zeros(1, dtype=torch.int64, device="cuda")
    want = jx.qk_norm_rope(q, k, v, caches[0], caches[1], pos, slot)
    got = jx.qk_norm_rope(odd(q), odd(k), odd(v), odd(caches[2]), caches[3], pos, slot)
    assert torch.equal(got, want) and torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])


def test_strides_that_differ_are_refused():
    p = Paged(BF, 4, 2, 64, 16, [100], [5], seed=1)
    p.k = p.k.permute(0, 2, 1, 3).contiguous().transpose(1, 2)
    with pytest.raises(AssertionError):
        p.run()
