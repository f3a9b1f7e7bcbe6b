"""What the compiler makes of the token operators' device code (runs without a GPU: it compiles only)."""
import os
import re
import subprocess

import pytest

from paper_1611_09482_amd import build as B

OPERATORS = ["fwg_embed.hip", "fwg_normq.hip", "fwg_matmulq.hip", "fwg_logprob.hip"]

# Every helper that writes vectors to rows, each in a kernel of its own.
PROBE = """
#include "fwg_ops_dev.h"
using namespace fwg::opd;
template <int N> __device__ void fill(float (&v)[N], const float *p) {
  for (int i = 0; i < N; ++i) v[i] = p[i];
}
extern "C" {
__global__ void f32_plain(const float *in, float *out) { float v[8]; fill(v, in); store<false>(out, v); }
__global__ void f32_stream(const float *in, float *out) { float v[8]; fill(v, in); store<true>(out, v); }
__global__ void bf16_plain(const float *in, uint16_t *out) { float v[12]; fill(v, in); store<false>(out, v); }
__global__ void bf16_stream(const float *in, uint16_t *out) { float v[12]; fill(v, in); store<true>(out, v); }
__global__ void bytes_plain(const uint32_t *in, int8_t *out) { store_bytes<false>(out, in[0], in[1]); }
__global__ void bytes_stream(const uint32_t *in, int8_t *out) { store_bytes<true>(out, in[0], in[1]); }
}
"""


def device_ir(source, out):
    subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-emit-llvm", "-o", out, source], check=True,
                   capture_output=True)
    with open(out) as f:
        return f.read()


def test_row_stores_promise_the_elements_alignment_only(tmp_path):
    """Rows start at any element, so no store to one may be compiled as if its address were a multiple of 16."""
    source = tmp_path / "probe.hip"
    source.write_text(PROBE)
    ir = device_ir(str(source), str(tmp_path / "probe.ll"))
    for name, element in [("f32_plain", 4), ("f32_stream", 4), ("bf16_plain", 2), ("bf16_stream", 2), ("bytes_plain", 1),
                          ("bytes_stream", 1)]:
        body = re.search(r"define [^\n]*@%s\(.*?\n}" % name, ir, re.S).group(0)
        stores = re.findall(r"^ *store .*?, align (\d+)", body, re.M)
        assert stores and all(int(a) <= element for a in stores), (name, stores)
        assert len(re.findall("!nontemporal", body)) == (len(stores) if name.endswith("stream") else 0), name


@pytest.mark.parametrize("name", OPERATORS)
def test_no_access_claims_more_alignment_than_its_type(name):
    r = subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-fsyntax-only", "-Werror=align-mismatch",
                                              os.path.join(B.CSRC, name)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]


def test_lanes_of_the_sort_see_each_others_places(tmp_path):
    """The radix sort's lanes read places in LDS that other lanes of the wave have just moved on: a wavefront fence has
    to stand between, or the compiler may exchange the two."""
    ir = device_ir(os.path.join(B.CSRC, "fwg_embed.hip"), str(tmp_path / "embed.ll"))
    body = re.search(r"define [^\n]*scatter_kernel.*?\n}", ir, re.S).group(0)
    assert 'syncscope("wavefront")' in body


def test_every_kernel_of_log_probs_is_reached(tmp_path):
    """Rows of one float32 batch are short rows, so the kernel that takes one batch a wave is there for bf16 only."""
    ir = device_ir(os.path.join(B.CSRC, "fwg_logprob.hip"), str(tmp_path / "logprob.ll"))
    names = set(re.findall(r"define [^\n]*@(\S*rows_kernelI\S*?)\(", ir))
    batches = sorted((n[n.index("rows_kernelI") + 12], re.search(r"Li(\d+)E", n).group(1)) for n in names)
    assert batches == [("f", "4"), ("f", "4"), ("t", "1"), ("t", "1"), ("t", "4"), ("t", "4")], names
