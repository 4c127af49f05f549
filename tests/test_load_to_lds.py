"""The load to LDS of the experts' products (csrc/expert_tiles.hpp) sets m0: the compiler has to know, or a value that it holds
there is lost.  A value is put into m0 before such a load and wanted there behind it."""
import os
import subprocess

from paper_2302_01425_amd import build

SOURCE = r"""
#include "%s"
extern "C" __global__ void probe(const char* from, uint32_t to) {
  uint32_t held;
  asm volatile("; set %%0" : "={m0}"(held));
  topk::load_to_lds(from, to);
  asm volatile("; use %%0" ::"{m0}"(held));
}
"""


def test_m0_is_declared(tmp_path):
    src, out = tmp_path / "probe.hip", tmp_path / "probe.s"
    src.write_text(SOURCE % os.path.join(build.CSRC, "expert_tiles.hpp"))
    subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", str(src), "-o", str(out)], check=True, capture_output=True)
    body = out.read_text()
    body = body[body.index("; set m0"):body.index("; use m0")]
    load = body.index("global_load_lds_dwordx4")
    assert "s_mov_b32 m0," in body[load:] or "v_readlane_b32 m0," in body[load:], body      # (it is put back)
