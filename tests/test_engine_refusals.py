"""A call of the engine that raises leaves its requests as they were: a caller that goes on after the error must not
attend over tokens whose K and V were never written."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_25523_amd import binding as B  # noqa: E402
from paper_2608_25523_amd import workloads as W  # noqa: E402
from paper_2608_25523_amd.engine import Engine  # noqa: E402
from paper_2608_25523_amd.rope import Rope, rope_frequencies  # noqa: E402

HQ, HKV, D, PAGES = 8, 2, 64, 12


def state(e):
    return ({r: p.tolist() for r, p in e.req_pages.items()}, dict(e.req_len), dict(e.req_agent), e.alloc.num_free())


def rows(n, heads, seed, device):
    x = np.random.default_rng(seed).standard_normal((n, heads, D)).astype(np.float32)
    return torch.from_numpy(W.bf16_round(x).view(np.int16)).to(device).view(torch.bfloat16)


def bookkeeping(rope=None):
    """An engine's tables and allocator without its device memory: what a call does before its first launch."""
    e = Engine.__new__(Engine)
    e.hq, e.hkv, e.d, e.num_pages, e.device = HQ, HKV, D, PAGES, "cpu"
    e.kv_format, e.rope, e.alloc = B.PFX_KV_E4M3, rope, B.Allocator(PAGES)
    e.pool = B.make_pool8(PAGES, HKV, D)
    e.prefix_len, e.resident = [16], {}
    e.req_pages = {5: e.alloc.alloc(1), 6: e.alloc.alloc(2)}
    e.req_len, e.req_agent = {5: 16, 6: 20}, {5: -1, 6: -1}
    return e


def test_refused_by_the_rotation():
    e = bookkeeping(Rope(rope_frequencies(D, device="cpu")))
    was = state(e)
    q, k = rows(2, HQ, 1, "cpu"), rows(2, HKV, 2, "cpu")
    for bad in ((q.float(), k, k), (q, k[:1], k), (q[:, :, ::2], k, k)):
        with pytest.raises(ValueError):
            e.decode([5, 6], *bad)
        assert state(e) == was
    with pytest.raises(ValueError):
        e.prefill(9, -1, q.float(), k, k)
    assert state(e) == was


def test_refused_for_want_of_pages():
    """The second request's pages are not there: the first one keeps its old length too."""
    e = bookkeeping()
    was = state(e)
    q = torch.zeros((1, HQ, D), dtype=torch.bfloat16)
    with pytest.raises(B.PfxError) as err:
        e.run([5, 6], [1, 16 * PAGES], q, q, q, B.PFX_MODE_EXTEND)
    assert err.value.code == B.PFX_ENOMEM and state(e) == was
    assert e.alloc.alloc(1).tolist() == [3]  # in the order in which they would have been handed out


def test_refused_for_a_request_named_twice():
    e = bookkeeping()
    was = state(e)
    q = torch.zeros((2, HQ, D), dtype=torch.bfloat16)
    with pytest.raises(B.PfxError):
        e.run([5, 5], [1, 1], q, q, q, B.PFX_MODE_DECODE)
    assert state(e) == was


@pytest.mark.gpu
@pytest.mark.parametrize("kv_format", [B.PFX_KV_BF16, B.PFX_KV_E4M3])
def test_goes_on_after_a_refusal(kv_format):
    """Refused calls in between change nothing of what the others return."""
    print(f"\n[gpu-case] engine with refused calls, format {kv_format}", flush=True)
    prefix = [tuple(W.bf16_round(np.random.default_rng(i).standard_normal((21, HKV, D)).astype(np.float32))
                    for i in (0, 1))]
    results = []
    for refusals in (False, True):
        e = Engine(PAGES, HQ, HKV, D, prefix, kv_format=kv_format, rope=Rope(rope_frequencies(D)))
        e.load(0)

        def call(f, *args, n, seed):
            q, k, v = (rows(n, h, 3 * seed + i, "cuda") for i, h in enumerate((HQ, HKV, HKV)))
            if refusals:
                was = state(e)
                bad = [(q.float(), k, v), (q, k.half(), v), (q, k.cpu(), v)]
                if kv_format == B.PFX_KV_E4M3:
                    bad += [(q, k, v.float()), (q, k, v[:, :1])]
                for x in bad:
                    with pytest.raises(ValueError):
                        f(*args, *x)
                    assert state(e) == was
            return f(*args, q, k, v)

        out = [call(e.prefill, 1, 0, n=19, seed=1), call(e.prefill, 2, -1, n=15, seed=2)]
        out += [call(e.decode, [1, 2], n=2, seed=3 + i) for i in range(3)]
        torch.cuda.synchronize()
        results.append([t.view(torch.uint8) for o in out for t in o])
    assert all(torch.equal(a, b) for a, b in zip(*results))
