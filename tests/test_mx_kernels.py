"""No kernel of the 4-bit operators and adjust_logits is compiled that no call launches (runs without a GPU: compiles only)."""
import os
import re
import subprocess

import pytest

from paper_1611_09482_amd import build as B


def kernels(name, out):
    """Sorted (kernel, template arguments) of a source's device code."""
    subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-o", out, os.path.join(B.CSRC, name)], check=True,
                   capture_output=True)
    with open(out) as f:
        mangled = re.findall(r"\.amdhsa_kernel (\S+)", f.read())
    found = []
    for m in mangled:
        kernel, args = re.match(r"_ZN3fwg\d(?:mx|mmx|adj)\d+([a-z]+_kernel)(?:I((?:[tf]|L[ib]\d+E)+)E)?E", m).groups()
        found.append((kernel, tuple({"t": "bf16", "f": "f32"}[t] if t else int(n)
                                    for t, n in re.findall(r"([tf])|L[ib](\d+)E", args or ""))))
    return sorted(found, key=str)


TYPES = ["bf16", "f32"]


def adjust():
    """Vocabularies up to 2,048 are one part; more go to blocks of 512 threads, a row's parts together or in turn."""
    return [("adjust_kernel", (t,) + k) for t in TYPES for k in [(256, 1, 0), (512, 2, 0), (512, 2, 1)]]


def mx():
    """Rows past the caches or not; norms by width, with an eps that hides small squares or not."""
    norms = [(64, 1), (64, 2), (256, 1), (256, 2), (1024, 1), (1024, 2), (1024, 4)]
    return ([("quant_kernel", (t, far)) for t in TYPES for far in (0, 1)] +
            [("norm_kernel", (t,) + n + (far, bare)) for t in TYPES for n in norms for far in (0, 1) for bare in (0, 1)])


def matmul():
    """Results of parts of k are float32; those past the caches come from large tiles."""
    return ([("pack_kernel", ())] + [("add_kernel", (t,)) for t in TYPES] +
            [("rows_kernel", (t,) + k) for t in TYPES for k in [(1, 1), (1, 2), (2, 1), (4, 1)]] +
            [("ring_kernel", (t, copied, sums)) for t, sums in [("bf16", 0), ("f32", 0), ("f32", 1)] for copied in (0, 1)] +
            [("tile_kernel", (t, copied) + k) for t in TYPES for copied in (0, 1) for k in [(0, 128), (0, 256), (1, 256)]])


@pytest.mark.parametrize("name,wanted", [("fwg_adjust.hip", adjust), ("fwg_mx.hip", mx), ("fwg_matmulmx.hip", matmul)])
def test_kernels_that_calls_launch(name, wanted, tmp_path):
    assert kernels(name, str(tmp_path / "k.s")) == sorted(wanted(), key=str)
