"""A step of the engine does not wait for the work before it on the stream."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_25523_amd import binding as B  # noqa: E402
from paper_2608_25523_amd import workloads as W  # noqa: E402
from paper_2608_25523_amd.engine import Engine  # noqa: E402
from paper_2608_25523_amd.rope import Rope, rope_frequencies  # noqa: E402

pytestmark = pytest.mark.gpu

HQ, HKV, D = 8, 2, 64


@pytest.mark.parametrize("kv_format", [B.PFX_KV_BF16, B.PFX_KV_E4M3])
def test_a_step_returns_before_the_work_in_front_of_it(kv_format):
    """Prefill and decode behind some 45 ms of products, with the same results as on an idle stream."""
    print(f"\n[gpu-case] engine step behind other work, format {kv_format}", flush=True)
    prefix = [tuple(W.bf16_round(np.random.default_rng(i).standard_normal((21, HKV, D)).astype(np.float32))
                    for i in (0, 1))]
    big = torch.ones((8192, 8192), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    qkv = [torch.randn((n, HQ + 2 * HKV, D), device="cuda", generator=g).to(torch.bfloat16) for n in (19, 1, 1, 1)]
    results = []
    for busy in (False, True):
        e = Engine(32, HQ, HKV, D, prefix, kv_format=kv_format, rope=Rope(rope_frequencies(D)))
        e.load(0)
        out = []
        for i, x in enumerate(qkv):
            parts = x.split([HQ, HKV, HKV], dim=1)
            torch.cuda.synchronize()
            before = torch.cuda.Event()
            for _ in range(60 if busy else 0):
                torch.mm(big, big)
            before.record()
            out.append(e.prefill(1, 0, *parts) if i == 0 else e.decode([1], *parts))
            if busy and i > 0:  # the first call of a process may load code
                assert not before.query(), "the call waited for the products in front of it"
        torch.cuda.synchronize()
        results.append([t.view(torch.uint8) for o in out for t in o])
    assert all(torch.equal(a, b) for a, b in zip(*results))
