"""dQ over long sequences runs beside the kernel for dK and dV and does not wait for what both read: what that rests on, in the source."""
import re

from paper_2603_06738_b200 import build

SOURCE = re.sub(r"//[^\n]*", "", (build.CSRC / "rib_cross_bwd_sm100.cu").read_text())


def part(begin, end):
    first = SOURCE.index(begin)
    return SOURCE[first:SOURCE.index(end, first)]


def test_dk_and_dv_start_it_behind_their_own_wait():
    kernel = part("rib_cross_bwd_dkv_kernel(", "struct SumTensor")
    assert kernel.count("cudaTriggerProgrammaticLaunchCompletion") == 1
    wait, start = (kernel.index(f"cuda{name}()") for name in ("GridDependencySynchronize", "TriggerProgrammaticLaunchCompletion"))
    assert wait < start and not kernel[wait:start].split(";")[1].strip()      # (the next statement)


def test_no_kernel_comes_between_them():
    launches = re.findall(r"launch_overtaking\((\w+)", part("cudaError_t launch_bwd(", "size_t cross_bwd_workspace"))
    assert launches == ["rib_cross_bwd_dkv_kernel", "rib_cross_bwd_dq_kernel"]


def test_its_reads_go_past_l1():
    decode = part("DqItem decode(", "template <int DP>")
    assert "__ldcg(p.lengths" in decode and "p.lengths[" not in decode
    kernel = part("rib_cross_bwd_dq_kernel(", "kKvThreads")
    assert "p.lengths" not in kernel
    assert not re.search(r"[=(]\s*p\.stats\[", kernel)


def test_its_last_cta_ends_behind_the_kernel_beside_it():
    kernel = part("rib_cross_bwd_dq_kernel(", "kKvThreads")
    assert "if (blockIdx.x == gridDim.x - 1) cudaGridDependencySynchronize();" in kernel and kernel.count("cudaGridDependencySynchronize") == 1
