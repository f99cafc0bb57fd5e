"""The hand-overs inside chunk_kernel, on the CPU: what no run can show, because it depends on timing."""
import os
import re

SOURCE = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_18139_b200", "csrc",
                           "chunk_kernel.cu")).read()


def test_tensor_memory_that_another_warpgroup_reads_is_fenced_on_both_sides():
    """Stream 0 reads stream 1's output block once merge_full has told it so: an mbarrier orders tensor memory only between a fence in front
    of the arrival and one behind the wait."""
    role = SOURCE[SOURCE.index("void softmax_rows"):SOURCE.index("chunk_kernel(const __grid_constant__")]
    arrival = role.index("mbar_arrive(ptx::smem_u32(&sh.merge_full))")
    wait = role.index("warp_wait(&sh.merge_full")
    reads = role.index("tmem_ld_32x16(to + kHeadDim")
    stores = [m.start() for m in re.finditer(r"tmem_(st|ld)_32x\d+\(t", role) if m.start() < arrival]
    assert max(stores) < role.rindex("tc_fence_before_sync()", 0, arrival)
    assert wait < role.index("tc_fence_after_sync()", wait) < reads
    assert role.rindex("tc_fence_before_sync()", 0, arrival) > role.index("if (!it.pair && g == 1)")
