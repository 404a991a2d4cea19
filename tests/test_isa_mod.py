"""Properties of the emitted gfx950 code of the kernels with a bias and with dropout that their synchronisation relies on: the same
that test_isa_invariants.py checks for the plain ones.  Cross-compiled here, no GPU needed."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2604_27124_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
UNITS = ("sigattn_rel_dropout_64", "sigattn_rel_128", "sigattn_dropout_128")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """(unit, name) -> instruction lines and bytes of scratch of each attention kernel."""
    out = tmp_path_factory.mktemp("isa")
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]

    def compile(unit):
        subprocess.run([B.hipcc(), *flags, "-I", os.path.join(ROOT, "include"), "-S", "--cuda-device-only", "-o", str(out / unit),
                        os.path.join(B.CSRC, unit + ".hip")], check=True, capture_output=True)

    with ThreadPoolExecutor(len(UNITS)) as pool:
        list(pool.map(compile, UNITS))
    result = {}
    for unit in UNITS:
        name = None
        for line in (out / unit).read_text().split("\n"):
            m = re.match(r"^(_Z\w+):", line)
            if m:
                name = (unit, m.group(1)) if "sigattn_mod" in m.group(1) else None
                if name:
                    result[name] = {"body": [], "scratch": None}
            elif name and re.match(r"^; ScratchSize: \d+", line):
                result[name]["scratch"] = int(line.split()[-1])
            elif name and result[name]["scratch"] is None:
                ins = line.split(";")[0].strip()
                if ins and (not ins.startswith(".") or ins.startswith(".LBB")):
                    result[name]["body"].append(ins)
    return result


def loops(name):
    """Passes over the streamed tiles."""
    return 2 if "sigattn_mod_bwd" in name[1] else 1


def test_every_kernel_is_looked_at(kernels):
    assert sorted(u for u, _ in kernels) == ["sigattn_dropout_128"] * 5 + ["sigattn_rel_128"] * 5 + ["sigattn_rel_dropout_64"] * 3
    assert all(k["scratch"] is not None and any(i.startswith("s_endpgm") for i in k["body"]) for k in kernels.values())


def test_tile_barrier_counts_its_reads(kernels):
    """Along every way that leads to a barrier with a partial wait, at least as many LDS operations follow the last LDS write as
    the wait lets stay in flight: then the writes have completed, since a wave's LDS operations complete in order.  (A scalar load,
    which counts on the same counter in any order, can only make the wait longer.)"""
    for name, k in kernels.items():
        body = k["body"]
        label = {ins[:-1]: i for i, ins in enumerate(body) if ins.endswith(":")}
        jumps = {}
        for i, ins in enumerate(body):
            m = re.match(r"s_c?branch\w* (\.LBB\w+)", ins)
            if m:
                jumps.setdefault(label[m.group(1)], []).append(i)

        def before(i):
            came = list(jumps.get(i, ()))
            if i > 0 and not re.match(r"s_branch |s_endpgm", body[i - 1]):
                came.append(i - 1)
            return came

        partial = 0
        for i, ins in enumerate(body):
            if ins != "s_barrier":
                continue
            w = i - 1
            while re.match(r"(v_|s_)(?!waitcnt|load|buffer_load|barrier|c?branch)", body[w]) and i - w < 8:
                w -= 1
            m = re.match(r"s_waitcnt (?:vmcnt\(\d+\) )?lgkmcnt\((\d+)\)$", body[w])
            if m is None:                                      # the wait of a __syncthreads() at the end of the blocks in front of it
                assert not re.match(r"s_waitcnt", body[w]), f"{name}: {body[w]!r} in front of a barrier"
                continue
            allowed = int(m.group(1))
            if allowed == 0:
                continue
            assert w == i - 1, f"{name}: instructions between a partial LDS wait and its barrier"
            partial += 1
            seen, todo = {}, [(w, 0)]
            while todo:
                at, reads = todo.pop()
                if seen.get(at, 99) <= reads:
                    continue
                seen[at] = reads
                for j in before(at):
                    assert body[j] != "s_barrier", f"{name}: no tile store between two barriers"
                    if body[j].startswith("ds_write"):
                        assert reads >= allowed, f"{name}: lgkmcnt({allowed}) but {reads} LDS operations follow a tile store"
                    else:
                        todo.append((j, reads + body[j].startswith("ds_")))
        assert partial == 4 * loops(name), f"{name}: {partial} tile barriers"


def test_no_packed_fp32_and_few_spills(kernels):
    for name, k in kernels.items():
        assert not any(re.match(r"v_pk_(add|mul|fma)_f32", i) for i in k["body"]), name
        # d = 128: the eight-wave dQ pass with a bias parks some registers a tile, the four-wave dK/dV pass some around its loop
        assert k["scratch"] <= (128 if "Li128E" in name[1] else 16), f"{name}: {k['scratch']} bytes"


def test_no_floating_point_atomics(kernels):
    for name, k in kernels.items():            # (the work mapping counts tiles with integer ones)
        assert not any(re.match(r"(global|flat|buffer)_atomic|ds_(pk_)?add\w*_(f|bf)", i) for i in k["body"]), name


def test_wide_stores_keep_their_data(kernels):
    """A store of more than two dwords reads its data registers a little later than it is issued; with a scalar offset the compiler does not
    count on that.  So no such store is followed at once by an instruction that writes them."""
    def registers(operand):
        m = re.match(r"v\[(\d+):(\d+)\]$|v(\d+)$", operand)
        return set() if m is None else set(range(int(m.group(1)), int(m.group(2)) + 1)) if m.group(1) else {int(m.group(3))}

    for name, k in kernels.items():
        ins = [i for i in k["body"] if not i.endswith(":")]
        for at, store in enumerate(ins):
            m = re.match(r"buffer_store_dwordx[34] (\S+), .*, s\d+ offen", store)
            if m is None:
                continue
            for after in ins[at + 1:at + 3]:
                if after.startswith("s_nop"):
                    break
                assert not (after.startswith("v_") and registers(after.split()[1].rstrip(",")) & registers(m.group(1))), f"{name}: {store} / {after}"
