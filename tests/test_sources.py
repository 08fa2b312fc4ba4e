"""Properties of the CUDA sources that no run can show (CPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2207_08393_b200", "csrc")


def test_no_read_only_loads_in_kernels_that_start_early():
    """Every kernel may be scheduled while the launch before it still writes what it will read (griddepcontrol.wait is its
    first statement), and a read-only load promises that the data stay as they are for the kernel's lifetime."""
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        for number, line in enumerate(open(os.path.join(CSRC, name)), 1):
            code = line.split("//")[0]
            assert not re.search(r"__ldg\b|__restrict__|ld\.global\.nc", code), "%s:%d" % (name, number)


def test_a_warp_barrier_stands_before_copies_into_slots_of_other_lanes():
    """Bricks: a lane copies 16 bytes, its own slot and its neighbour's, so the neighbour has to have read its slot before.  A
    shuffle in between orders no memory accesses; only __syncwarp() does."""
    code = [line.split("//")[0] for line in open(os.path.join(CSRC, "dc_brick.cuh"))]
    reads = [i for i, line in enumerate(code) if "u[m] = e[m * W];" in line]
    copies = [i for i, line in enumerate(code) if "cp_async16(e - odd" in line]
    assert len(reads) == len(copies) == 1 and reads[0] < copies[0]
    assert any("__syncwarp();" in line for line in code[reads[0]:copies[0]])


def test_products_that_add_to_one_sum_have_one_shape():
    """Matrix instructions follow each other in the order of their issue only if they share the place of their sums and the shape."""
    for name in ("ortho_gemm.cuh", "ortho_resident.cuh"):
        code = "".join(line.split("//")[0] + "\n" for line in open(os.path.join(CSRC, name)))
        products = re.findall(r"tc::product\(([^;]*)\);", code)
        assert products and all(p.split(",")[-2].strip() == "what" for p in products), name
        shapes = re.findall(r"what = tc::instruction\((\w+), ", code)
        assert len(shapes) == code.count("tc::instruction("), name
        for shape in shapes:
            assert shape in ("BLOCK", "R"), name


def test_sums_are_split_by_sizes_alone():
    """Replicas of a model on several GPUs compute the same bits: how many clusters the current GPU holds decides nothing but whether it takes
    those of more than eight blocks."""
    code = "".join(line.split("//")[0] + "\n" for line in open(os.path.join(CSRC, "ortho_ops.cu")))
    assert code.count("cudaOccupancyMaxActiveClusters") == 1
    body = code[code.index("static int clusters_at_once"):code.index("cudaOccupancyMaxActiveClusters")]
    assert "if (ranks <= RESIDENT_PORTABLE) return at_once[ranks];" in body


def test_a_launch_that_gave_up_waiting_leaves_nan():
    """The torch layer drops the workspace and its status word, so results have to tell.  No run of a working kernel waits in vain: what every sum is
    multiplied with on its way out of tensor memory is NaN after a wait that did."""
    read = lambda name: "".join(line.split("//")[0] + "\n" for line in open(os.path.join(CSRC, name)))
    assert "unit_of(bool failed) { return failed ? __int_as_float(0x7fffffff) : 1.f / SCALE; }" in read("ortho_common.cuh")
    gemm, resident = read("ortho_gemm.cuh"), read("ortho_resident.cuh")
    assert gemm.index("failed = __syncthreads_or(failed);") < gemm.index("unit = unit_of(failed);")
    out = gemm[gemm.index("unit = unit_of(failed);"):]
    assert out.index("read_sums(half, v);") < out.index(": v[j]) * unit;") < out.index("(sum + sum_at(row, c0 + j)) = ")
    assert "v[j] = (v[j] + u[j]) * unit_of(failed);" in resident and resident.count("tc::read_columns(") == 2
    assert resident.count("if (threadIdx.x == 0 && !failed)") == resident.count("what = tc::instruction(")
