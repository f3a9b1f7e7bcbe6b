"""What the compiler makes of the 4-bit operators' and adjust_logits' device code (runs without a GPU: it compiles only)."""
import os
import re
import subprocess

import pytest

from paper_1611_09482_amd import build as B

SOURCES = ["fwg_mx.hip", "fwg_matmulmx.hip", "fwg_adjust.hip"]


def device_asm(name, out):
    subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-o", out, os.path.join(B.CSRC, name)], check=True,
                   capture_output=True)
    with open(out) as f:
        return f.read()


@pytest.mark.parametrize("name", SOURCES)
def test_no_access_claims_more_alignment_than_its_type(name):
    r = subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-fsyntax-only", "-Werror=align-mismatch",
                                              os.path.join(B.CSRC, name)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]


def kernels(asm):
    """{kernel: (its code, registers, scratch bytes)}"""
    found = {}
    for name in re.findall(r"\.amdhsa_kernel (\S+)", asm):
        body = asm[asm.index("\n%s:" % name):]
        about = asm[asm.index(".amdhsa_kernel " + name):]
        found[name] = (body[:body.index("s_endpgm")], int(re.search(r"next_free_vgpr (\d+)", about).group(1)),
                       int(re.search(r"private_segment_fixed_size (\d+)", about).group(1)))
    return found


def test_products_keep_their_sums_in_registers(tmp_path):
    """A register spilled inside a loop over stages would wait, when it is read back, for the copies on their way to LDS."""
    for name, (body, registers, scratch) in kernels(device_asm("fwg_matmulmx.hip", str(tmp_path / "m.s"))).items():
        assert scratch <= 16 and registers <= 256, (name, registers, scratch)
        assert len(re.findall("scratch_(?:load|store)", body)) <= 4, name  # a pair around the loops, not one in them


def test_results_past_the_caches_where_rows_are_whole_lines(tmp_path):
    """Two stores that differ only in this would be merged into one without it: the variants are kernels of their own."""
    tiles = {n: b for n, (b, _, _) in kernels(device_asm("fwg_matmulmx.hip", str(tmp_path / "m.s"))).items() if "tile_kernel" in n}
    stores = {n: re.findall(r"global_store_dwordx4[^\n]*", b) for n, b in tiles.items()}
    streamed = [n for n, s in stores.items() if any(x.endswith(" nt") for x in s)]
    assert len(streamed) == 4 and all(all(x.endswith(" nt") for x in stores[n]) for n in streamed), stores


def test_the_ring_waits_for_what_it_needs_only(tmp_path):
    """Three stages are on their way to LDS while one is multiplied: a wait for all of them inside the loop would end that."""
    rings = {n: b for n, (b, _, _) in kernels(device_asm("fwg_matmulmx.hip", str(tmp_path / "m.s"))).items()
             if re.search("ring_kernelI.Lb1", n)}
    assert len(rings) == 3
    for name, body in rings.items():
        loops = [b for b in re.split(r"\n(?=\.LBB)", body) if "Loop Header" in b and b.count("s_barrier") >= 4]
        assert len(loops) == 1, name
        waits = re.findall(r"vmcnt\((\d+)\)", loops[0])
        assert waits == ["8"] * 4 and loops[0].count("global_load_lds_dwordx4") == 16, (name, waits)
