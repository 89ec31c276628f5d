"""Norms of heads whose squares leave the range of fp32, against fp64."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_25523_amd import binding as B  # noqa: E402
from test_gpu_rope import check, frequencies  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,rotary,interleaved", [(128, 128, False), (64, 32, True), (64, 0, False)])
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-27, 1e-6])
def test_heads_of_every_magnitude(d, rotary, interleaved, eps):
    """One head a power of two from bf16's least to its largest, others of several in one head."""
    print(f"\n[gpu-case] norms from 2^-133 to 2^127, d={d} rotary={rotary} eps={eps}", flush=True)
    rng = np.random.default_rng(d + rotary)
    # Below 2^-90 of every magnitude; above, of those whose squares fp32 holds.
    exps = np.arange(-133, 128 if eps < 2.0 ** -90 else 59)
    tokens, hq, hkv = len(exps), 3, 2
    x = rng.uniform(0.5, 1.0, (tokens, hq + hkv, d)) * rng.choice([-1.0, 1.0], (tokens, hq + hkv, d))
    x = np.ldexp(x, exps[:, None, None])
    x[:, 1, ::2] = 0.0                                          # half of the head
    x[:, 2] = 0.0
    x[:, 2, 5] = np.ldexp(1.0, exps)                            # one value alone
    x[:, 4] = np.ldexp(x[:, 4], -rng.integers(0, 40, (tokens, d)))  # magnitudes far apart
    qk = torch.from_numpy(x).to(torch.float32).to(torch.bfloat16).cuda()
    qk[:, 4, 0] = torch.where(qk[:, 4, 0] == 0, 2.0 ** -133, qk[:, 4, 0].float()).to(torch.bfloat16)  # not all zeros
    qk[:, 0, 0] = torch.where(qk[:, 0, 0] == 0, 2.0 ** -133, qk[:, 0, 0].float()).to(torch.bfloat16)
    qk[:, 1, 1] = torch.where(qk[:, 1, 1] == 0, 2.0 ** -133, qk[:, 1, 1].float()).to(torch.bfloat16)
    qk[:, 3, 0] = torch.where(qk[:, 3, 0] == 0, 2.0 ** -133, qk[:, 3, 0].float()).to(torch.bfloat16)
    q, k = qk[:, :hq], qk[:, hq:]
    w = torch.from_numpy(rng.standard_normal((2, d))).to(torch.bfloat16).cuda()
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda") * 37
    freq = frequencies(rotary).cuda()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    B.pfx_qk_norm_rope(q, k, pos, freq, qo, ko, w[0], w[1], eps, interleaved)
    B.pfx_sync_check()
    assert torch.isfinite(qo.float()).all() and torch.isfinite(ko.float()).all()
    eps = float(np.float32(eps))
    check(qo, q, pos, freq, w[0], eps, interleaved, "q")
    check(ko, k, pos, freq, w[1], eps, interleaved, "k")


def test_infinities_and_nan_stay_in_their_heads():
    print("\n[gpu-case] heads with infinities and NaN", flush=True)
    d = 64
    x = torch.randn((3, 4, d), device="cuda").to(torch.bfloat16)
    clean = x.clone()
    x[0, 1, 7], x[1, 2, 0], x[2, 3, 63] = float("inf"), float("nan"), float("-inf")
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    pos, freq = torch.arange(3, dtype=torch.int32, device="cuda"), frequencies(d).cuda()
    outs = []
    for t in (x, clean):
        o = torch.empty_like(t)
        B.pfx_qk_norm_rope(t, t[:, :1], pos, freq, o, torch.empty_like(t[:, :1]), w, None, 0.0)
        outs.append(o)
    B.pfx_sync_check()
    bad = torch.zeros((3, 4), dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[1, 2] = bad[2, 3] = True
    assert torch.equal(outs[0][~bad], outs[1][~bad])
    assert torch.isnan(outs[0][1, 2]).all() and torch.isnan(outs[0][0, 1, 7]) and torch.isnan(outs[0][2, 3, 63])
