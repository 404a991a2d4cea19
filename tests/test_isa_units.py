"""Properties of the emitted gfx950 code of every translation unit of the library: how wide stores are addressed, what test_isa_mod.py checks for the units that it
leaves out, and what goes through scratch from tile to tile.  Cross-compiled here, no GPU needed."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

import test_isa_mod as mod_checks
from paper_2604_27124_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
UNITS = [s[:-len(".hip")] for s in B.SOURCES]


@pytest.fixture(scope="module")
def units(tmp_path_factory):
    """(unit, kernel) -> its instruction lines and labels."""
    out = tmp_path_factory.mktemp("isa")
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]

    def compile(unit):
        subprocess.run([B.hipcc(), *flags, "-I", os.path.join(ROOT, "include"), "-S", "--cuda-device-only", "-o", str(out / unit),
                        os.path.join(B.CSRC, unit + ".hip")], check=True, capture_output=True)

    with ThreadPoolExecutor(min(4, len(UNITS))) as pool:
        list(pool.map(compile, UNITS))
    result = {}
    for unit in UNITS:
        name = None
        for line in (out / unit).read_text().split("\n"):
            m = re.match(r"^(_Z\w+):", line)
            if m:
                name = (unit, m.group(1))
                result[name] = []
            elif line.startswith(".Lfunc_end"):
                name = None
            elif name:
                ins = line.split(";")[0].strip()
                if ins and (not ins.startswith(".") or ins.startswith(".LBB")):
                    result[name].append(ins)
    return {name: body for name, body in result.items() if any(i.startswith("s_endpgm") for i in body)}


@pytest.fixture(scope="module")
def mod_kernels(units):
    """The attention kernels with a bias and dropout, all six units."""
    return {name: {"body": body} for name, body in units.items() if "sigattn_mod" in name[1]}


def scalar_offset_stores(body):
    """Stores of more than two dwords whose offset is in a scalar register.  Such a store reads its data registers a little later than it is issued, and the
    compiler leaves no wait before the next instruction writes them."""
    return [i for i in body if re.match(r"buffer_store_dwordx[34] v\[\d+:\d+\], v\d+, s\[\d+:\d+\], (s\d+|m0|vcc_lo|vcc_hi|ttmp\d+)( |$)", i)]


def test_the_check_sees_such_a_store():
    bad = "buffer_store_dwordx4 v[4:7], v9, s[8:11], s3 offen sc1"
    assert scalar_offset_stores(["s_nop 0", bad, "buffer_store_dwordx4 v[4:7], v9, s[8:11], 0 offen offset:1024", "buffer_store_dword v4, v9, s[8:11], s3 offen"]) == [bad]


def test_no_wide_store_has_a_scalar_offset(units):
    assert {u for u, _ in units} >= {u for u in UNITS}
    wide = 0
    for name, body in units.items():
        wide += sum(i.startswith("buffer_store_dwordx4") for i in body)
        assert not scalar_offset_stores(body), f"{name}: {scalar_offset_stores(body)[:3]}"
    assert wide > 300                                           # what the library's epilogues are made of


def test_barriers_of_all_units(mod_kernels):
    assert sorted({u for u, _ in mod_kernels}) == sorted(u for u in UNITS if u.endswith(("_64", "_128")))
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
        parks = "sigattn_modILi1ELi128ELi1ELi8E" in name[1] and "ELb1EL" in name[1]
        for l in range(mod_checks.loops(name)):
            spills = sum(i.startswith("scratch_") for i in k["body"][ends[4 * l]:ends[4 * l + 3]])
            assert spills <= (80 if parks and name[0] == "sigattn_rel_dropout_128" else 16 if parks else 0), f"{name}: {spills}"
