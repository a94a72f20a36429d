"""The kernels of ordered histories as they were compiled: no vector register spilled, and no copy of a vector register where a branch
of some lanes ends, before the other lanes are back.

Such a copy reaches only the lanes that took the branch; where the others read it later as an address they go astray.  The compiler was seen to
make one when it ran out of vector registers around a divergent branch, so both are looked for in what was built."""
import os
import re
import struct
import subprocess

import pytest

from paper_2112_02194_amd import binding as als

TOOLS = "/opt/rocm/llvm/bin"
KERNELS = ("walk_all_kernel", "walk_last_kernel", "pieces_kernel", "join_kernel", "recur_step_kernel", "clip_norm_kernel", "clip_scale_kernel", "beam_kernel",
           "reorder_kernel")


def code_objects(path):
    """The gfx950 code objects of a library built by hipcc: one per translation unit, in bundles one after the other."""
    data = open(path, "rb").read()
    magic, at, out = b"__CLANG_OFFLOAD_BUNDLE__", 0, []
    while (at := data.find(magic, at)) >= 0:
        (count,), place = struct.unpack_from("<Q", data, at + len(magic)), at + len(magic) + 8
        for _ in range(min(count, 8)):
            offset, size, length = struct.unpack_from("<QQQ", data, place)
            name = data[place + 24:place + 24 + length]
            place += 24 + length
            if b"gfx950" in name and size:
                out.append(data[at + offset:at + offset + size])
        at += len(magic)
    return out


@pytest.fixture(scope="module")
def units(tmp_path_factory):
    if not os.path.exists(als.LIB_PATH):
        pytest.skip("library not built")
    if not os.path.exists(os.path.join(TOOLS, "llvm-readelf")):
        pytest.skip("no tools to read code objects")
    found = []
    for i, code in enumerate(code_objects(als.LIB_PATH)):
        if any(name.encode() in code for name in KERNELS):
            path = str(tmp_path_factory.mktemp("code") / f"{i}.o")
            with open(path, "wb") as f:
                f.write(code)
            found.append(path)
    assert len(found) == 4  # recur, sum_rows, clip and beam
    return found


def test_no_vector_register_is_spilled(units):
    kernels = 0
    for path in units:
        notes = subprocess.run([os.path.join(TOOLS, "llvm-readelf"), "--notes", path], capture_output=True, text=True, check=True).stdout
        for block in re.split(r"\n\s+- \.agpr_count", notes)[1:]:
            name = re.search(r"\.name:\s+(\S+)", block).group(1)
            kernels += 1
            assert re.search(r"\.vgpr_spill_count:\s+(\d+)", block).group(1) == "0", name
            assert re.search(r"\.private_segment_fixed_size:\s+(\d+)", block).group(1) == "0", name
    assert kernels > 100


def copies_before_lanes_return(listing):
    """(kernel, copies) wherever vector registers are copied between the head of a block that a branch over an empty set of lanes leads to
    and the instruction that brings the other lanes back."""
    found, kernel, lines = [], None, {}
    for line in listing.splitlines():
        if (m := re.match(r"^<(_Z\w+)>:$", line)):
            kernel = m.group(1)
        lines.setdefault(kernel, []).append(line.split("//")[0].strip())
    for kernel, body in lines.items():
        ends = {m.group(1) for line in body if (m := re.match(r"s_cbranch_execz\s+(L\d+)$", line))}
        copies = None  # None: not at the head of such a block
        for line in body:
            if (m := re.match(r"<(L\d+)>:$", line)):
                copies = [] if m.group(1) in ends else None
            elif copies is None:
                continue
            elif line.startswith("s_or_b64 exec, exec"):
                if copies:
                    found.append((kernel, copies))
                copies = None
            elif re.match(r"v_mov_b\d+\S* v\S+, v|v_accvgpr|scratch_", line):
                copies.append(line)
            elif re.match(r"s_(branch|cbranch|endpgm)", line):
                copies = None
    return found


def test_what_is_looked_for():
    """A block that ends a branch of some lanes, with a copy before the lanes are back, behind them, and none."""
    def listing(block):
        return "<_Zkernel>:\n\ts_and_saveexec_b64 s[0:1], vcc\n\ts_cbranch_execz L1\n\tv_add_f32_e32 v0, v1, v2\n<L1>:\n" + block + "\ts_endpgm\n"
    back, copy = "\ts_or_b64 exec, exec, s[0:1]   // 00: 01\n", "\tv_mov_b64_e32 v[52:53], v[66:67]   // 02: 03\n"
    assert copies_before_lanes_return(listing(copy + back)) == [("_Zkernel", ["v_mov_b64_e32 v[52:53], v[66:67]"])]
    assert copies_before_lanes_return(listing(back + copy)) == []
    assert copies_before_lanes_return(listing("\tv_mov_b32_e32 v3, 0\n" + back)) == []  # a constant is no copy
    assert copies_before_lanes_return(listing(copy)) == []  # nothing is brought back here


def test_no_copy_before_the_lanes_are_back(units):
    for path in units:
        listing = subprocess.run([os.path.join(TOOLS, "llvm-objdump"), "-d", "--symbolize-operands", path], capture_output=True, text=True, check=True).stdout
        listing = re.sub(r"(?m)^[0-9a-f]+ (<\w+>:)$", r"\1", listing)
        assert "s_cbranch_execz" in listing and re.search(r"s_cbranch_execz\s+L\d+", listing)
        assert copies_before_lanes_return(listing) == []
