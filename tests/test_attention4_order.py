"""Tensor memory, registers and launches of decoding from 4-bit pages, read from its source (CPU only), and how
its calls are cut up, from their workspaces."""
import os
import re

import pytest

from paper_2608_25332_gb300 import build as pbuild

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_25332_gb300", "csrc")
TC, PLAIN = "attention_decode4_tc.cu", "attention_decode4.cu"


def source(file):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())


def body(file, kernel):
    src = source(file)
    i = src.index("{", re.search(r"__global__[^{;]*\b" + kernel + r"\(", src).end())
    depth = 0
    for j in range(i, len(src)):
        depth += (src[j] == "{") - (src[j] == "}")
        if depth == 0:
            return src[i:j]


def test_tensor_memory_is_held_before_the_next_kernels_may_start():
    b = body(TC, "attn4_prefix_tc")
    alloc = b.index("tmem_alloc(")
    assert alloc < b.index("__syncthreads()", alloc) < b.index("pdl_allow_next()")
    assert "pdl_wait_prior()" not in b  # launched behind all work before it
    assert b.count("return;") == 0      # every thread gets to the release of the tensor memory
    assert b.rindex("__syncthreads()") < b.index("tmem_dealloc(")


def test_the_joining_kernel_waits_for_the_prefix_through_the_own_keys():
    """it waits for the kernel before it alone; that one ends behind the prefix's, in each way out"""
    b = body(PLAIN, "attn4_kernel")
    wait = "if (!kPrefix && first) pdl_wait_prior();"
    assert b.count("return;") == 1 and b.count(wait) == 2 and wait in b[:b.index("return;")][-60:] and b.rstrip().endswith(wait)
    assert body(PLAIN, "attn4_join").lstrip("{ \n").startswith("pdl_wait_prior();")
    # its inputs are there when it starts early: only a kernel of the same call, launched plainly, lies in between
    src = source(PLAIN)
    assert "if (!kPrefix && plan.n_pre > 0)" in src and src.count("launch_pdl(") == 2 and "launch_pdl" not in source(TC)


def test_register_split_is_covered_by_the_launch():
    src = source(TC)
    launch, soft, mma, expand = map(int, re.search(
        r"kLaunchRegs = (\d+), kSoftRegs = (\d+), kMmaRegs = (\d+), kExpandRegs = (\d+);", src).groups())
    assert 256 * soft + 128 * mma + 256 * expand <= 640 * launch and soft > launch > max(mma, expand)
    assert "at.numRegs != kLaunchRegs" in src  # and checked against the build
    # whole warpgroups change their registers together: 0-7, 8-11, 12-19
    assert "kSoftWarps = 8, kMmaWarp = 8, kExpandWarp = 12" in src and "kThr = 640" in src


def test_named_barriers_are_met_by_all_of_their_warps():
    """barriers have no limit on their wait: the expanding warps meet theirs once a tile, whatever their waits gave"""
    b = body(TC, "attn4_prefix_tc")
    loop = b[b.index("for (int t = 0; t < nt; ++t) {", b.index("kExpandRegs")):]
    loop = loop[:loop.index("if (!live) ctl.fail = 1;")]
    assert loop.count("expand_sync(") == 1 and "break" not in loop and "continue" not in loop
    assert b.count("expand_sync(") == 1


def test_commits_are_waited_for():
    """nothing arrives at a barrier of a block that has ended: operands are given back only to a tile that follows"""
    b = body(TC, "attn4_prefix_tc")
    assert "if (lead && live && t < nt) tc_commit(&ctl.empty[1]);" in b and "if (t + 1 < nt) tc_commit(&ctl.empty[0]);" in b
    assert b.count("tc_commit(&ctl.empty") == 2


@pytest.fixture(scope="module")
def L():
    pbuild.build()
    from paper_2608_25332_gb300 import provip
    return provip.lib()


def parts(L, B, H_q, H_kv, kv, prefix, dtype):
    """parts a row, from the workspace: 128 sums and a log-sum-exp each, both rounded up"""
    ws, rows = L.provip_decode_attention4_workspace_size(B, H_q, H_kv, kv, prefix, dtype), B * H_q
    up = lambda n: -(-n // 256) * 256
    return next((n for n in range(0, 1100) if ws <= up(n * rows * 512) + up(n * rows * 4) + 256), None)


@pytest.mark.parametrize("dtype", [0, 1])
def test_no_parts_where_a_wave_is_full(L, dtype):
    for B in (9, 16, 128, 4096):
        assert parts(L, B, 32, 32, 2339, 0, dtype) in (0, 1)  # 288 units of three times 152, or more
    assert parts(L, 1, 32, 32, 211, 0, dtype) in (0, 1)       # too few keys
    assert parts(L, 1, 28, 4, 9379, 0, dtype) == 37           # 256 keys a part at least


@pytest.mark.parametrize("dtype", [0, 1])
def test_parts_are_few_enough_to_be_joined(L, dtype):
    for B, H_q, H_kv, kv, prefix in ((1, 1, 1, 2 ** 31 - 600, 0), (1, 1, 1, 2 ** 30, 2 ** 30 - 1), (1, 17, 1, 10 ** 6, 10 ** 6),
                                     (65535, 1, 1, 1, 1), (3, 8, 8, 0, 5000), (64, 28, 4, 512, 9251)):
        n = parts(L, B, H_q, H_kv, kv, prefix, dtype)
        assert n is not None and n <= 768
