"""Rules of plans over the 8-bit pool that differ from the bf16 pool's, because the kernels do."""

from __future__ import annotations

import numpy as np
import pytest

pytest.importorskip("torch")

import kv8_cases as KC  # noqa: E402
from paper_2608_25523_amd import binding as B  # noqa: E402


def plan8(hq, hkv, d, prefix_len, reqs, **kw):
    b = KC.batch(1, hq, hkv, d, prefix_len, reqs)
    return B.plan_from_batch(B.make_pool8(b.num_pages, hkv, d), b, kv_format=B.PFX_KV_E4M3, **kw)


@pytest.mark.parametrize("agents,prefix,reqs", [(1, 2048, 64), (4, 8192, 32), (4, 10000, 16), (2, 4096, 56)])
def test_decode_pieces_fit_the_chip_at_head_dim_64(agents, prefix, reqs):
    """decode8_kernel<64> has 148 registers: three workgroups a compute unit, 768 at once.  Where pieces of 16 steps
    are no more than that, a shorter length must not make them more."""
    batch = (32, 8, 64, [prefix] * agents, [(i % agents, 64 + 7 * i % 449, 1) for i in range(reqs)])
    fixed, auto = (plan8(*batch, **kw).stats().num_decode_pieces for kw in (dict(piece_steps=16), {}))
    longest = plan8(*batch, piece_steps=64).stats().num_decode_pieces
    assert longest <= 768, "the batch fits at some length"
    assert auto <= max(768, fixed), (auto, fixed)


def test_registers_behind_the_rule(tmp_path):
    """The figure the rule stands on, from the compiler: above 128 registers and up to 168, three waves a SIMD."""
    import os
    import re
    import subprocess
    hipcc = "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    from paper_2608_25523_amd.build import FLAGS, HERE, ROOT
    out = tmp_path / "k.s"
    subprocess.run([hipcc, *[f for f in FLAGS if f not in ("-shared", "-fPIC")], "-S", "--cuda-device-only", "-I",
                    os.path.join(ROOT, "include"), os.path.join(HERE, "csrc", "pfx_kv8.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    waves = {}
    for name, body in re.findall(r"\.globl\s+(\S*decode8_kernel\S*).*?; Kernel info:(.*?)\.text", out.read_text(), re.S):
        waves[re.search(r"ILi(\d+)E", name).group(1)] = int(re.search(r"; Occupancy: (\d+)", body).group(1))
    assert waves == {"64": 3, "128": 2}, waves


def cut_bytes(batch, **kw):
    """Workspace that the pieces of cut extend blocks take: what a plan has over one of whole blocks with the same
    decode pieces."""
    auto = plan8(*batch, **kw)
    for steps in range(1, 65):
        whole = plan8(*batch, piece_steps=steps)
        same = [(s.num_decode_pieces, s.num_partial_rows) for s in (auto.stats(), whole.stats())]
        if same[0] == same[1]:
            return auto.workspace_bytes() - whole.workspace_bytes()
    raise AssertionError("no fixed length gives the same decode pieces")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,prefix,decode", [(300, 4096, 8), (1200, 2048, 32), (32, 4096, 16)])
def test_extend_blocks_and_decode_pieces_plan_apart(d, rows, prefix, decode):
    """They run in launches of their own: a mixed batch is cut as its two halves are."""
    prompt = [(0, rows, rows)]
    steps = [(0, 64 + 13 * i % 300, 1) for i in range(decode)]
    mixed, alone = cut_bytes((32, 8, d, [prefix], prompt + steps)), cut_bytes((32, 8, d, [prefix], prompt))
    assert abs(mixed - alone) <= 1024, (mixed, alone)  # sections are rounded up to 256 bytes
    counts = [plan8(32, 8, d, [prefix], r).stats().num_decode_pieces for r in (prompt + steps, steps)]
    assert counts[0] == counts[1], counts


@pytest.mark.parametrize("batch", [(8, 2, 64, [128], [(0, 32, 32)] * 4), (32, 8, 128, [400], [(0, 32, 32)] * 3),
                                   (4, 4, 128, [], [(-1, 20, 20)])])
def test_whole_extend_blocks_take_no_pieces_table(batch):
    """The table lets the append ride in the extend launch, which no 8-bit launch does: the workspace holds the plan's
    other sections and no more."""
    plan = plan8(*batch)
    s = plan.stats()
    assert s.num_decode_pieces == 0 and s.num_extend_items > 0
    size = [plan.export(i).size * 4 for i in (0, 1, 8, 2)] + [4 * s.num_tokens, plan.export(4).size * 4]
    assert plan.workspace_bytes() == sum((x + 255) // 256 * 256 for x in size)
