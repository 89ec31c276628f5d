"""The 8-bit attention kernels over long key ranges, at real sizes and next to the largest values they take, against the
fp64 oracle.

A wave of an extend block holds the page ids of its next 128 pages (2048 keys) and asks for more as it goes: the
prefixes here take more, with odd page counts, so that a half step shifts the table from the suffix on."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv8_cases as KC  # noqa: E402
from oracle.attention import bf16_bits_to_f64  # noqa: E402
from paper_2608_25523_amd import binding as B  # noqa: E402
from paper_2608_25523_amd import workloads as W  # noqa: E402

pytestmark = pytest.mark.gpu


def announce(msg):
    print(f"\n[gpu-case] {msg}", flush=True)


def random_pool(pages, hkv, d, seed):
    """An 8-bit pool of N(0, 1) keys and values, its descriptor and its bytes on the host."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    src = torch.randn((2, pages, hkv, 16, d), device="cuda", generator=g).to(torch.bfloat16)
    t = [torch.zeros((pages, hkv, w), dtype=torch.uint8, device="cuda") for w in (16 * d, 16 * d, 2)]
    pool = B.make_pool8(pages, hkv, d, *t)
    ws = torch.empty(B.pfx_page_quantize_workspace_bytes(pages) + 256, dtype=torch.uint8, device="cuda")
    ids = np.arange(pages, dtype=np.int32)
    B.pfx_page_quantize(pool, B.make_pool(pages, hkv, d, src[0], src[1]), ids, ids, ws)
    B.pfx_sync_check()
    return t, pool, [x.cpu().numpy() for x in t]


class OnPool:
    """A batch whose tokens the pool holds already, and queries of it."""

    def __init__(self, b, seed):
        self.b = b
        rng = np.random.default_rng(seed)
        self.q = W.bf16_round(rng.standard_normal((b.num_tokens, b.num_q_heads, b.head_dim)).astype(np.float32))

    def attend(self, pool, workspace=None, **kw):
        plan = B.plan_from_batch(pool, self.b, kv_format=B.PFX_KV_E4M3, **kw)
        plan.upload(*([] if workspace is None else [workspace(plan)]))
        q = torch.from_numpy(self.q.view(np.int16)).cuda().view(torch.bfloat16)
        o, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
        B.pfx_attention8(pool, plan, q, o, lse)
        B.pfx_sync_check()
        return o.view(torch.int16).cpu().numpy().view(np.uint16), lse.cpu().numpy()

    reference = KC.Host8.reference


# (hq, hkv, d, prefix lengths, requests): 4100 keys are 257 pages, 2053 are 129.
LONG = {
    "one-prompt": (4, 1, 128, [4100], [(0, 40, 40)]),
    "one-prompt-d64": (4, 1, 64, [4100], [(0, 37, 37)]),
    "odd-pages": (2, 2, 128, [2053, 4099], [(0, 70, 70), (1, 33, 20), (-1, 70, 70)]),
    "odd-pages-d64": (8, 2, 64, [2053, 4099], [(0, 20, 20), (1, 49, 33)]),
    "long-suffix": (8, 1, 128, [17], [(0, 4500, 23)]),
    "no-prefix": (4, 1, 64, [], [(-1, 6001, 19)]),
    "mixed": (8, 2, 128, [4100, 37], [(0, 300, 1), (0, 40, 40), (1, 17, 1), (0, 31, 1), (1, 2500, 18)]),
}


@pytest.mark.parametrize("how", ["cut", "whole", "small-workspace"])
@pytest.mark.parametrize("name", sorted(LONG))
def test_long_key_ranges(name, how):
    announce(f"long keys, {name}, {how}")
    b = KC.batch(51, *LONG[name])
    _, pool, host = random_pool(b.num_pages, b.num_kv_heads, b.head_dim, 52)
    case = OnPool(b, 53)
    kw = {}
    plans = [B.plan_from_batch(pool, b, kv_format=B.PFX_KV_E4M3, piece_steps=x).workspace_bytes() for x in (0, 64)]
    assert plans[0] > plans[1] + 2 * 128 * b.head_dim * 4, "the automatic plan cuts the blocks"
    if how == "whole":
        kw = dict(piece_steps=64)
    elif how == "small-workspace":
        # Room for the decode pieces' states of this very plan, none for those of cut blocks.
        part = 2 * 128 * b.head_dim * 4
        kw = dict(workspace=lambda plan: torch.empty(plan.workspace_bytes() - part + 256, dtype=torch.uint8,
                                                     device="cuda"))
    worst = KC.check(*case.attend(pool, **kw), case.reference(host), f"{name} {how}")
    announce(f"long keys, {name}, {how}: {worst:.2f} of the bound")


def test_pieces_far_into_the_page_table():
    """Two requests, many KV heads: pieces that start past the first 64 table entries and run over several windows."""
    announce("few pieces of long blocks")
    b = KC.batch(61, 16, 8, 128, [8200], [(0, 300, 300), (0, 20, 20)])
    _, pool, host = random_pool(b.num_pages, 8, 128, 62)
    case = OnPool(b, 63)
    o, lse = case.attend(pool)
    ref = case.reference(host, only=[1])
    KC.check(o, lse, ref, "the short request")
    whole = case.attend(pool, piece_steps=16)
    KC.check(*whole, ref, "the short request, whole blocks")
    # The long one, row by row in the 2-norm: the two ways it is summed in, apart by what each may be off (2^-8 of it
    # for both, as half a step of bf16 in P and in O is 2^-9 in the root mean square).
    x, y = (bf16_bits_to_f64(t[0]) for t in ((o,), whole))
    assert (np.linalg.norm(x - y, axis=2) <= 2.0 ** -7 * np.linalg.norm(x, axis=2)).all()
    assert np.max(np.abs(lse - whole[1])) <= 2.0 ** -12


def test_large_decode_batch_against_fp64():
    """64 requests of 4 agents over 2048 tokens each: the first and last request and one of each agent, every element
    against the oracle; and all rows against a plan of other pieces."""
    announce("64 decode requests, 4 agents, against fp64")
    rng = np.random.default_rng(41)
    b = W.make_batch(41, num_q_heads=32, num_kv_heads=8, head_dim=128, num_pages=3000, prefix_len=[2048] * 4,
                     agent=np.arange(64) % 4, suffix_len=rng.integers(64, 512, 64), n_rows=np.ones(64, np.int32))
    _, pool, host = random_pool(3000, 8, 128, 64)
    case = OnPool(b, 65)
    o, lse = case.attend(pool, mode=B.PFX_MODE_DECODE)
    KC.check(o, lse, case.reference(host, only=[0, 5, 30, 43, 63]), "64 requests")
    other = case.attend(pool, mode=B.PFX_MODE_DECODE, piece_steps=5)
    x, y = bf16_bits_to_f64(o), bf16_bits_to_f64(other[0])
    # Row by row in the 2-norm: either's probabilities and its own rounding to bf16 are off by half a step of 2^-8 at
    # most, 2^-9 in the root mean square, 2^-8 together for both plans; a key of 2300 that were lost or counted twice
    # would change the row by 1 / sqrt(2300) = 2^-5.6.
    assert (np.linalg.norm(x - y, axis=2) <= 2.0 ** -7 * np.linalg.norm(x, axis=2)).all()
    assert np.max(np.abs(lse - other[1])) <= 2.0 ** -12


@pytest.mark.parametrize("name,reqs", [("decode", [(0, 600, 1), (-1, 900, 1)]), ("extend", [(0, 40, 40), (-1, 900, 33)])])
def test_values_at_the_end_of_the_range(name, reqs):
    """max |V| times a row's keys just below 2^119: sums of probabilities of up to 2^8 stay finite.  All keys alike, whose
    sums are the largest, but for those that a kernel takes first (extend blocks the first ones, decode waves the last),
    7.5 lower in log2, from which the running maximum does not move."""
    announce(f"values near 2^119 / keys, {name}")
    d, prefix = 128, 1000
    keys = prefix + max(r[1] for r in reqs)
    b = KC.batch(71, 4, 1, d, [prefix], reqs)
    top = 2.0 ** np.floor(np.log2(2.0 ** 119 / keys))
    n = b.num_pages
    k, v = np.zeros((n, 1, 16, d)), np.full((n, 1, 16, d), top)
    k[..., 0] = 1.0
    for pages in list(b.prefix_pages) + list(b.suffix_pages):
        k[pages[:4], ..., 0] = 0.0
        k[pages[-9:], ..., 0] = 0.0
    v[..., 64:] *= np.where(np.random.default_rng(72).random(v[..., 64:].shape) < 0.9, 1.0, -0.5)
    t = [torch.from_numpy(W.bf16_round(x.astype(np.float32)).view(np.int16)).cuda().view(torch.bfloat16) for x in (k, v)]
    p8 = [torch.zeros((n, 1, w), dtype=torch.uint8, device="cuda") for w in (16 * d, 16 * d, 2)]
    pool = B.make_pool8(n, 1, d, *p8)
    ids = np.arange(n, dtype=np.int32)
    ws = torch.empty(B.pfx_page_quantize_workspace_bytes(n) + 256, dtype=torch.uint8, device="cuda")
    B.pfx_page_quantize(pool, B.make_pool(n, 1, d, *t), ids, ids, ws)
    B.pfx_sync_check()
    case = OnPool(b, 73)
    q = np.zeros(case.q.shape, np.float32)
    q[..., 0] = 7.5 * np.log(2.0) * np.sqrt(d)
    case.q = W.bf16_round(q)
    for kw in ({}, dict(piece_steps=64), dict(piece_steps=2)):
        o, lse = case.attend(pool, **kw)
        assert np.isfinite(bf16_bits_to_f64(o)).all()
        KC.check(o, lse, case.reference([x.cpu().numpy() for x in p8]), f"{name} {kw}")
