"""Order within a warp in the attention kernels, read from their source (CPU only)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_25332_gb300", "csrc")
FILES = ["attention_tc.cu", "attention_decode_tc.cu"]


def code(file):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())


@pytest.mark.parametrize("file", FILES)
def test_a_units_slot_is_handed_back_behind_a_warp_barrier(file):
    """One lane hands the slot back for the warp: the other lanes' reads of it come before a
    barrier of the warp, which is the statement before."""
    src = code(file)
    found = [m.start() for m in re.finditer(r"if \(lane == 0\) mbar_arrive\(&ctl\.u_empty", src)]
    assert len(found) == (3 if file == "attention_tc.cu" else 2)
    for at in found:
        assert src[:at].rstrip().endswith("__syncwarp();"), src[at - 200:at + 60]


@pytest.mark.parametrize("file", FILES)
def test_no_lane_leaves_a_round_before_the_warps_tensor_memory_access(file):
    """A lane that goes to the loop's next round by itself would meet an access that the whole warp
    has to make together (.sync.aligned) alone: rounds with one have no condition of a lane's own
    that ends them."""
    src = code(file)
    for m in re.finditer(r"\bfor \([^;{]*;[^;{]*;[^{]*\) \{", src):
        depth, j = 0, src.index("{", m.start())
        for j in range(j, len(src)):
            depth += (src[j] == "{") - (src[j] == "}")
            if depth == 0:
                break
        body = src[m.end():j]
        if "tmem_ld" in body or "tmem_st" in body:
            # (raise, live and the unit's fields are the warp's)
            ends = re.findall(r"if \(([^;{}]*)\) (?:continue|break|return)\b", body)
            for cond in ends:
                assert "row_live" not in cond and "lane" not in cond, (file, cond)


def test_rows_computed_again_follow_the_warps_stores():
    """Rows that are not finite are stored by one set of lanes and again by another: a barrier of
    the warp lies between."""
    for file in ("attention_tc.cu", "attention_simt.cu"):
        src = code(file)
        again = [m.start() for m in re.finditer(r"attn_row_plain<[^;]*\(a, ", src)]
        assert again
        for at in again:
            vote = src.rindex("__ballot_sync(", 0, at)
            assert src[:src.rindex(";", 0, vote)].rstrip().endswith("__syncwarp()"), file


@pytest.mark.parametrize("file", FILES)
def test_waits_outlast_rows_that_are_computed_again(file):
    """A warp that computes rows again by the definition may take longer than a wait's limit (a
    microsecond a key and row): the others' waits start again while it gets on."""
    src = code(file)
    drain = src.index("void drain(")
    roles = src[:drain] + src[src.index("\n}\n", drain):]
    assert not re.search(r"\bmbar_wait\(", roles), "waits without the sign of rows under way"
    assert "attn_row_plain" not in src or re.search(r"attn_row_plain<[^;]*&?(?:ctl\.)?beat\)", src)
    tc = code("attention_tc.cuh")
    wait = tc[tc.index("bool wait_over("):tc.index("bool warp_wait(")]
    # gives up only where the last sign of them is a whole limit ago too (read before the time is,
    # so that it is never ahead of it)
    assert re.search(r"last = \*[^;]*\(beat\), now = global_timer_ns\(\);", wait)
    assert re.search(r"if \(\(long long\)\(now - t0\) <= most \|\| \(long long\)\(now - last\) <= most\) return false;", wait)
    assert "&& wait_over(t0, err, beat)) return false;" in wait and wait.count("return false;") == 2
    plain = code("attention.cuh")
    plain = plain[plain.index("attn_row_plain("):]
    assert re.search(r"& 63\) == 0\) [^;]*\(beat\) = global_timer_ns\(\);", plain[:plain.index("\n}\n")])


@pytest.mark.parametrize("file", FILES)
def test_a_flag_in_shared_memory_is_read(file):
    """what a role leaves for the others is read by one of them"""
    src = code(file)
    struct = src[src.index("struct Ctl {"):]
    struct = struct[:struct.index("\n};")]
    for name in re.findall(r"\b(?:int|uint32_t|float) (\w+)(?:\[\w+\])*;", struct):
        uses = re.findall(r"\bctl\." + name + r"\b(?!\s*(?:\[[^\]]*\])*\s*=[^=])", src)
        assert uses, f"{file}: {name} is written and never read"


@pytest.mark.parametrize("file", FILES)
def test_a_block_outlasts_what_it_has_issued(file):
    """Where a wait gives up, loads into the block's shared memory and products in its tensor memory
    may still be under way. The warps that issued them wait for them (once more with a limit)
    before the release of tensor memory and the block's end."""
    src = code(file)
    end = src[src.rindex("if (ctl.fail) {"):]
    assert re.match(r"if \(ctl\.fail\) \{\s*drain(?:<NQ>)?\(ctl, a\.err\);\s*__syncthreads\(\);\s*\}\s*if \(warp == 0\) tmem_dealloc\(", end)
    assert src[:src.rindex("if (ctl.fail) {")].rstrip().endswith("__syncthreads();")
    drain = src[src.index("void drain("):]
    drain = drain[:drain.index("\n}\n")]
    # the products: by the lane that issued them
    assert re.search(r"if \(elect_one\(\)\) \{\s*tc_commit\(&ctl\.mma_done\);\s*mbar_wait\(&ctl\.mma_done, 0, err\);", drain)
    assert "const bool lead = elect_one();" in src
    # the loads: every barrier that one of them signals
    loads = set(re.findall(r"tma_load_\dd\([^;]*&ctl\.(\w+)(?:\[[^\]]*\])?\);", src)) | ({"full"} if "uint64_t* full = &ctl.full[" in src else set())
    assert len(loads) == 2
    for bar in loads:
        assert re.search(r"mbar_wait\(&ctl\." + bar + r"\b", drain), bar
    # and every role that gives up says so
    roles = src[src.index("__global__", src.index("void drain(")):]
    assert len(re.findall(r"if \(!live\) ctl\.fail = 1;", roles)) == (3 if file == "attention_tc.cu" else 2)
    assert len(re.findall(r"if \(failed\) ctl\.fail = 1;", roles)) == 1
