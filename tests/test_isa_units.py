"""Properties of the gfx950 code of every kernel in the library as it is built: how wide stores are addressed, what test_isa_mod.py checks for some of the units, and
what goes through scratch from tile to tile.  No GPU needed."""
import os
import re
import shutil
import subprocess

import pytest

import test_isa_mod as mod_checks
from paper_2604_27124_amd import binding
from paper_2604_27124_amd import build as B


@pytest.fixture(scope="module")
def units(tmp_path_factory):
    """Kernel -> its instruction lines and labels (in the form that the compiler's own listing has), out of the library as it is built."""
    binding.load()                                              # builds it if it is not there
    out = tmp_path_factory.mktemp("isa")
    lib = shutil.copy(B.LIB, out / "lib.so")
    objdump = os.path.join(os.path.dirname(os.path.realpath(B.hipcc())), "..", "llvm", "bin", "llvm-objdump")
    if not os.path.exists(objdump):
        objdump = "/opt/rocm/llvm/bin/llvm-objdump"
    subprocess.run([objdump, "--offloading", lib], check=True, capture_output=True, cwd=out)
    result = {}
    for image in sorted(p for p in os.listdir(out) if p.endswith("gfx950")):
        text = subprocess.run([objdump, "-d", "--symbolize-operands", "--no-show-raw-insn", "--no-leading-addr", image], check=True, capture_output=True,
                              text=True, cwd=out).stdout
        body = None
        for line in text.split("\n"):
            line = line.split("//")[0].strip()
            m = re.match(r"<(\w+)>:$", line)
            if m and m.group(1).startswith("_Z"):
                body = result.setdefault(m.group(1), [])
            elif m:
                body.append(f".LBB_{m.group(1)}:")
            elif line and body is not None:
                body.append(re.sub(r"^(s_c?branch\w*) (L\d+)$", r"\1 .LBB_\2", line))
    return {name: body for name, body in result.items() if any(i.startswith("s_endpgm") for i in body)}


@pytest.fixture(scope="module")
def mod_kernels(units):
    """The attention kernels with a bias and dropout: (a name for its messages, the kernel's own) -> its code."""
    return {("lib", name): {"body": body} for name, body in units.items() if "sigattn_mod" in name}


def scalar_offset_stores(body):
    """Stores of more than two dwords whose offset is in a scalar register.  Such a store reads its data registers a little later than it is issued, and the
    compiler leaves no wait before the next instruction writes them."""
    return [i for i in body if re.match(r"buffer_store_dwordx[34] v\[\d+:\d+\], v\d+, s\[\d+:\d+\], (s\d+|m0|vcc_lo|vcc_hi|ttmp\d+)( |$)", i)]


def test_the_check_sees_such_a_store():
    bad = "buffer_store_dwordx4 v[4:7], v9, s[8:11], s3 offen sc1"
    assert scalar_offset_stores(["s_nop 0", bad, "buffer_store_dwordx4 v[4:7], v9, s[8:11], 0 offen offset:1024", "buffer_store_dword v4, v9, s[8:11], s3 offen"]) == [bad]


def test_no_wide_store_has_a_scalar_offset(units):
    for kernel in ("sigattn_onepassE", "sigattn_pair_bwd", "sigattn_half_bwd", "sigattn_bwd_kernel", "sigattn_mod_bwd", "sigattn_rel_few", "sigattn_rel_table"):
        assert any(kernel in name for name in units), kernel
    wide = 0
    for name, body in units.items():
        wide += sum(i.startswith("buffer_store_dwordx4") for i in body)
        assert not scalar_offset_stores(body), f"{name}: {scalar_offset_stores(body)[:3]}"
    assert wide > 300                                           # what the library's epilogues are made of


def test_barriers_of_all_units(mod_kernels):
    # three kernels at d = 64 and five at d = 128, each with the bias, dropout and both
    for bias, drop in (("1", "0"), ("0", "1"), ("1", "1")):
        assert sum(f"ELb{bias}ELb{drop}EE" in name for _, name in mod_kernels) == 8
    assert len(mod_kernels) == 24
    mod_checks.test_tile_barrier_counts_its_reads(mod_kernels)
    mod_checks.test_no_floating_point_atomics(mod_kernels)
    mod_checks.test_wide_stores_keep_their_data(mod_kernels)
    for name, k in mod_kernels.items():
        assert not any(re.match(r"v_pk_(add|mul|fma)_f32", i) for i in k["body"]), name


def tile_barriers(body):
    """Places of the barriers that end a streamed tile: those with a partial wait for LDS in front, four a pass."""
    return [i for i, ins in enumerate(body) if ins == "s_barrier" and re.match(r"s_waitcnt (?:vmcnt\(\d+\) )?lgkmcnt\([1-9]\d*\)$", body[i - 1])]


def test_registers_stay_in_registers_from_tile_to_tile(mod_kernels):
    """Scratch instructions in three tiles, between the four tile barriers of a pass.  The eight-wave dQ pass at d = 128 with a bias has 256 registers for its
    tiles, the sums and (with dropout) the generator, and parks some in every tile (6 with the bias alone, 69 with both); no other pass does."""
    for name, k in mod_kernels.items():
        ends = tile_barriers(k["body"])
        assert len(ends) == 4 * mod_checks.loops(name)
        parks = "sigattn_modILi1ELi128ELi1ELi8E" in name[1] and "ELb1ELb" in name[1]
        for l in range(mod_checks.loops(name)):
            spills = sum(i.startswith("scratch_") for i in k["body"][ends[4 * l]:ends[4 * l + 3]])
            assert spills <= (80 if parks and "ELb1ELb1EE" in name[1] else 16 if parks else 0), f"{name}: {spills}"
