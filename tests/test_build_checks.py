"""What a build refuses: kernels whose compiled form touches a register while its LDS read is in flight."""
import os

import pytest

from paper_2404_00509_amd import build, lds_reads

KERNEL = """#include <hip/hip_runtime.h>
#include "matmul.hpp"
__global__ void probe(float* out) {{
  __shared__ float lds[1024];
  lds[threadIdx.x] = out[threadIdx.x];
  __syncthreads();
  float __attribute__((ext_vector_type(4))) v;
  asm volatile("ds_read_b128 %0, %1" : "=v"(v) : "v"((unsigned)threadIdx.x * 4u & ~15u) : "memory");
  {wait}
  asm volatile("" : "+v"(v));
  out[threadIdx.x] = v.x + v.y;
}}
"""


def _compile(tmp_path, wait):
    source = tmp_path / "probe.hip"
    source.write_text(KERNEL.format(wait=wait))
    (tmp_path / "matmul.hpp").write_text("")
    build.compile_source(str(source), str(tmp_path / "probe.hip.o"))
    return tmp_path / "probe.hip.o"


def test_a_read_that_is_waited_for_is_built(tmp_path):
    assert os.path.getsize(_compile(tmp_path, 'asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");')) > 0


def test_a_read_that_is_used_too_early_is_refused(tmp_path):
    with pytest.raises(RuntimeError, match="in flight"):
        _compile(tmp_path, "")


def test_the_check_finds_the_reads_or_refuses():
    body = "probe:\n\t;;#ASMSTART\n\tds_read_b128 v[4:7], v9\n\t;;#ASMEND\n{}\ts_endpgm\n\t.size\tprobe, 1\n"
    assert lds_reads.check(body.format("\ts_waitcnt lgkmcnt(0)\n\tv_mov_b32_e32 v4, v5\n"), "probe") == 1
    with pytest.raises(RuntimeError, match="v_mov_b32_e32 v4, v8"):
        lds_reads.check(body.format("\tv_mov_b32_e32 v4, v8\n\ts_waitcnt lgkmcnt(0)\n"), "probe")
    with pytest.raises(RuntimeError, match="no LDS read"):
        lds_reads.check("probe:\n\ts_endpgm\n\t.size\tprobe, 1\n", "probe")


def test_the_sources_with_the_main_loop_are_checked():
    checked = [s for s in build.SOURCES if '#include "matmul.hpp"' in open(os.path.join(build.CSRC, s)).read()]
    assert checked == ["class_loss.hip", "embed_grad.hip"]
