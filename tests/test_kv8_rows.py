"""Plans without query rows over the 8-bit pool: their calls take None for the rows, as the C calls take NULL."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import kv8_cases as KC  # noqa: E402
from paper_2608_25523_amd import binding as B  # noqa: E402


def plan_of(reqs):
    b = KC.batch(3, 8, 2, 64, [20], reqs)
    t = [torch.zeros((b.num_pages, 2, w), dtype=torch.uint8) for w in (1024, 1024, 2)]
    if torch.cuda.is_available():
        t = [x.cuda() for x in t]
    pool = B.make_pool8(b.num_pages, 2, 64, *t)
    return t, pool, B.plan_from_batch(pool, b, kv_format=B.PFX_KV_E4M3)


def test_rows_of_a_plan_with_some_are_needed():
    _, pool, plan = plan_of([(0, 9, 1), (-1, 5, 0)])
    x = torch.zeros((1, 8, 64), dtype=torch.bfloat16)
    for args in ((None, None), (x, None), (None, x)):
        with pytest.raises(ValueError, match="contiguous bf16"):
            B.pfx_append_kv8(pool, plan, *args)
        with pytest.raises(ValueError, match="contiguous bf16"):
            B.pfx_attention8(pool, plan, *args)
        with pytest.raises(ValueError, match="contiguous bf16"):
            B.pfx_step8(pool, plan, x, x, *args)


@pytest.mark.gpu
@pytest.mark.parametrize("reqs", [[], [(0, 9, 0), (-1, 5, 0)]])
def test_no_rows_at_all(reqs):
    print(f"\n[gpu-case] calls of a plan without rows, requests {reqs}", flush=True)
    t, pool, plan = plan_of(reqs)
    plan.upload()
    empty = torch.zeros((0, 8, 64), dtype=torch.bfloat16, device="cuda")
    for x in (None, empty):
        B.pfx_append_kv8(pool, plan, x, x)
        B.pfx_attention8(pool, plan, x, x)
        B.pfx_step8(pool, plan, x, x, x, x)
    B.pfx_sync_check()
    assert not any(x.any() for x in t)


def test_pool_descriptors_refuse_tensors_that_do_not_hold_the_pool():
    k, v, s = (torch.zeros((5, 2, w), dtype=torch.uint8) for w in (1024, 1024, 2))
    ok = B.make_pool8(5, 2, 64, k, v, s)
    assert (ok.k_pages, ok.v_pages, ok.scales) == (k.data_ptr(), v.data_ptr(), s.data_ptr())
    B.make_pool8(4, 2, 64, k[1:], v[:4], s)  # room behind the pool
    for bad in ((k[1:], v, s), (k, v[:, :1], s), (k, v, s[:4]), (k.int(), v, s), (k, v, s.float()),
                (k, torch.zeros((5, 1024, 2), dtype=torch.uint8).transpose(1, 2), s)):
        with pytest.raises(ValueError, match="contiguous uint8"):
            B.make_pool8(5, 2, 64, *bad)
    with pytest.raises(ValueError, match="contiguous uint8"):
        B.make_pool8(5, 2, 128, k, v, s)
