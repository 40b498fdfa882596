"""What the sources of the routing, the norm and the products in 8 bits have to keep, where no run of them would show that it does not."""
import re

from test_g4_source import code, early_units


def test_kernels_wait_for_the_stream_before_they_read():
    """They start under the kernels ahead of them: each of them waits for the stream's order, once, before anything but its own shared
    memory is touched.  (That none of them reads by the read-only path is tested with the other kernels that start early.)"""
    assert {"rms_norm.cu", "route.cu", "i8_gemm.cu"} <= set(early_units())
    for name in ("rms_norm.cu", "route.cu", "i8_gemm.cuh"):
        kernels = re.split(r"__global__", code(name))[1:]
        assert kernels
        for body in kernels:
            assert body.count("wait_for_previous();") == 1, name
            ahead = body[body.index("{"):body.index("wait_for_previous();")]
            assert "p." not in ahead.replace("p.steps", "").replace("p.ftiles", "").replace("p.ttiles", "").replace("p.width", ""), name
            assert "tma_load" not in ahead and "pair_load" not in ahead and "bulk_load" not in ahead and "codes" not in ahead[1:], name


def test_every_wait_is_bounded():
    """No loop polls a barrier without a limit: waits go by short_wait or count."""
    for name in ("rms_norm.cu", "i8_gemm.cuh"):
        text = code(name)
        for m in re.finditer(r"mbar_try_wait", text):
            assert "wait_limit" in text[text.rfind("for (", 0, m.start()):m.end()], name
        assert "while (!" not in text


def test_threads_of_a_block_leave_the_ring_together():
    """The gradients' ring: a thread whose wait ran out still comes to the barrier, which tells all of them."""
    text = code("rms_norm.cu")
    loop = text[text.index("bool ok = short_wait(&full[at.s]"):]
    assert loop.index("if (!__syncthreads_and(ok)) break;") < loop.index("load(row + (int64_t)stages")
    assert "break" not in loop[:loop.index("__syncthreads_and")] and "return" not in loop[:loop.index("__syncthreads_and")]


def test_exponentials_are_taken_from_the_library():
    for name in ("route.cu", "rms_norm.cu", "i8_gemm.cuh"):
        assert "__expf" not in code(name) and "ex2.approx" not in code(name)
