"""Tensor memory and launches of the attention behind the pruning, read from its source (CPU
only), and how its calls are cut up, from their workspaces."""
import os
import re

import pytest

from paper_2608_25332_gb300 import build as pbuild

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_25332_gb300", "csrc")


def body(file, kernel):
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())
    m = re.search(r"__global__[^{;]*\b" + kernel + r"\(", src)
    i = src.index("{", m.end())
    depth = 0
    for j in range(i, len(src)):
        depth += (src[j] == "{") - (src[j] == "}")
        if depth == 0:
            return src[i:j]


@pytest.mark.parametrize("file,kernel", [("attention_tc.cu", "attn_tc"), ("attention_decode_tc.cu", "attn_keys_tc")])
def test_tensor_memory_is_held_before_the_next_kernel_may_start(file, kernel):
    """The own keys' kernel may start beside the prefix's, which by then holds its tensor memory
    in every CTA; neither waits for the other before it has its own."""
    b = body(file, kernel)
    alloc = b.index("tmem_alloc(")
    assert alloc < b.index("__syncthreads()", alloc) < b.index("pdl_allow_next()")
    assert "pdl_wait_prior()" not in b[:b.index("tmem_dealloc(")]


def test_own_keys_kernel_completes_after_the_prefix():
    """the joining kernel waits for the kernel before it alone"""
    b = body("attention_decode_tc.cu", "attn_keys_tc")
    assert "pdl_wait_prior()" in b[b.index("tmem_dealloc("):]


def test_register_split_is_covered_by_the_launch():
    src = open(os.path.join(CSRC, "attention_tc.cu")).read()
    m = re.search(r"kSoftRegs = NQ == 2 \? (\d+) : (\d+), kRestRegs = NQ == 2 \? (\d+) : (\d+);", src)
    soft2, soft1, rest2, rest1 = map(int, m.groups())
    # launched with 65536 / threads rounded down to eight: 168 for 384 threads, 128 for 2 x 256
    assert 256 * soft2 + 128 * rest2 <= 384 * 168 and 128 * soft1 + 128 * rest1 <= 256 * 128
    assert "at.numRegs * F::kThreads < F::kSoftRegs" in src  # and checked against the build


def test_named_barriers_are_met_by_a_fixed_number_of_warps():
    """barriers have no limit on their wait: the four softmax warps of the own keys' kernel leave
    their loop by a common vote only"""
    b = body("attention_decode_tc.cu", "attn_keys_tc")
    soft = b[b.index("bool failed = false;"):]
    assert "failed = soft_any(failed);" in soft and "if (failed || x.g < 0) break;" in soft
    assert soft[:soft.index("tmem_dealloc(")].count("return;") == 0


@pytest.fixture(scope="module")
def L():
    pbuild.build()
    from paper_2608_25332_gb300 import provip
    return provip.lib()


def test_no_parts_where_units_fill_the_gpu(L):
    ws = L.provip_prompt_attention_workspace_size
    assert ws(8 * 1091, 8, 32, 32, 1091, 1091, 0, 1, 0) == 0     # 1280 units of two row tiles
    assert ws(9379, 1, 28, 4, 9379, 9379, 0, 1, 0) == 0
    assert ws(48, 1, 32, 32, 48, 211, 0, 1, 0) == 0              # too few keys to share out
    assert ws(128, 1, 28, 4, 128, 9379, 0, 1, 0) > 0             # few rows, many keys


def test_decode_workspace(L):
    ws = L.provip_decode_attention_workspace_size
    rows, head = 64 * 28, 512 + 4
    # pieces of the spans' cuts: two a CTA at most, for a group's heads
    assert ws(32, 32, 32, 1091, 0, 1, 0) <= 2 * 304 * head + 304 * 8 + 33 * 8 + 5 * 256
    assert ws(64, 28, 4, 512, 9251, 1, 0) >= rows * head * 2
    assert ws(64, 28, 4, 0, 0, 1, 0) > 0
