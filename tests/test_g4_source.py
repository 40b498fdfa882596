"""What the source of the kernels on 4-bit weights has to keep, where no run of them would show that it does not."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2106_09886_b200" / "csrc"


def code(name):
    """A source file without its comments."""
    text = (CSRC / name).read_text()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def with_headers(name, seen=None):
    """A source file and the files of its own folder that it includes."""
    seen = set() if seen is None else seen
    if name not in seen and (CSRC / name).exists():
        seen.add(name)
        for other in re.findall(r'#include "([^"]+)"', code(name)):
            with_headers(other, seen)
    return seen


def early_units():
    return sorted(p.name for p in CSRC.glob("*.cu") if any("wait_for_previous();" in code(f) for f in with_headers(p.name) if f != "tc_ptx.cuh"))


def test_kernels_that_start_early_read_memory_coherently():
    """A kernel under programmatic stream serialization starts while the kernel ahead of it may still write what it will read.
    That memory is not read-only for the kernel's whole life, so no load may take the read-only path, neither by __ldg nor by
    a const __restrict__ parameter from which the compiler may infer it."""
    units = early_units()
    assert {"g4_rows.cu", "g4_stage.cu", "g4_tensor_fwd.cu", "g4_tensor_data.cu", "expert_wgrad.cu"} <= set(units)
    for unit in units:
        for name in with_headers(unit):
            for word in ("__ldg", "__restrict__", ".nc"):
                assert word not in code(name), f"{name} (in {unit}): {word}"


def test_every_kernel_that_starts_early_waits():
    """And each of them waits for the stream's order, all its threads, before its first role begins."""
    for name in ("g4_rows.cu", "g4_stage.cu", "g4_tensor.cuh", "expert_wgrad.cu"):
        kernels = re.split(r"__global__", code(name))[1:]
        assert kernels
        for body in kernels:
            assert body.count("wait_for_previous();") == 1, name
            ahead = body[:body.index("wait_for_previous();")]
            assert "offsets[" not in ahead and "expert_slot" not in ahead and "SlotCursor" not in ahead and "load(" not in ahead, name


def test_few_row_ring_is_released_behind_its_last_use():
    """An arrival on a stage's barrier does not wait for shared-memory loads in flight, so it must come after the instructions
    that use their values.  The compiler keeps that order only among volatile statements: the matrix instruction and every load
    of its operands are, and the arrival follows them."""
    text = code("g4_rows.cu")
    mma = re.search(r"void mma_16x8x16\(.*?\n\}", text, flags=re.S).group(0)
    assert mma.count("mma.sync") == 2 and len(re.findall(r"\basm\s+volatile\s*\(\s*\"mma\.sync", mma)) == 2
    kernel = text[text.index("g4_rows_kernel("):]
    assert "reinterpret_cast<const uint4 *>(smem" not in kernel
    assert kernel.index("lds_128(") < kernel.index("mma_16x8x16<T>(") < kernel.index("arrive_local(&empty")
    assert re.search(r"asm volatile\(\"ld\.shared\.v4", code("tc_ptx.cuh"))


def test_few_rows_barriers_are_reached_by_warps_that_gave_up():
    """The multiplying warps meet at barriers around each set of converted columns.  A warp whose bounded wait ran out must still
    come to every one of them, or the others would wait there without a limit: the loop that holds the barriers goes by the
    sizes alone, only the one inside it stops early."""
    text = code("g4_rows.cu")
    outer = re.search(r"for \(int t0 = first;([^;]*);", text)
    assert outer and outer.group(1).strip() == "t0 < last"
    body = text[outer.end():text.index("float *sums", outer.end())]
    inner = body.index("for (int t = 0; ok && t < here;")
    ahead, behind = body[:inner], body[body.index("s.next(C_STAGES);", inner):]
    assert ahead.count("multiplying_warps_sync();") == 2 and behind.count("multiplying_warps_sync();") == 1
    assert "break" not in ahead and "break" not in behind and "return" not in body


def test_items_of_a_grouped_product_are_bounded_whatever_the_offsets_hold():
    """Offsets are read on the device and may decrease, against the contract; 4096 experts that all claim every one of 2^23 - 1 rows
    make 2^30 blocks of 32 rows, times the tiles of features more than an int counts.  Every role's loop over items ends at a
    bound that the host has checked, so no item number wraps and no row is computed from one that did."""
    experts, rows, tile = 4096, 2 ** 31 // 256 - 1, 32
    assert experts // 2 * -(-rows // tile) * (4096 // 128) > 2 ** 31            # every second expert, 4096 features
    text = code("g4_tensor.cuh")
    loops = re.findall(r"for \(int t = first_work;([^;]*);", text)
    assert len(loops) == 3 and all(c.strip() == "t < p.items && !stop()" for c in loops)
    assert re.search(r"g4_stages\(items < p\.items \? items : p\.items,", text)
    assert text.index("work > 0x3FFFFFFFll") < text.index("p.items = (int)work;")
