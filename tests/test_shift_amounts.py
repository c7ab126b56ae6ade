"""No kernel shifts 64 bits by a number in the last of its vector registers: such a shift (by v255 of 256) has taken another
number here.  The compiler does not see to it for this target, so the built code is looked over."""
import concurrent.futures
import os
import re
import subprocess

import paper_2003_06324_amd as g
from paper_2003_06324_amd import build
from test_wide_store_data import _code_objects


def _last_registers(notes):
    """{kernel: number of the last vector register that its waves are given} of a code object's notes"""
    last, count = {}, None
    for line in notes.splitlines():
        m = re.match(r"\s*(?:- )?\.(symbol|vgpr_count|name):\s+'?([^\s']+)'?", line)
        if m and m.group(1) == "symbol":
            count = m.group(2)[:-len(".kd")]
        elif m and m.group(1) == "vgpr_count":
            last[count] = (int(m.group(2)) + 7) // 8 * 8 - 1
    return last


def _shifts(listing, last):
    """(64-bit shifts by a vector register, those by the kernel's last one) of a disassembly"""
    shifts, bad, kernel = 0, [], ""
    for line in listing.splitlines():
        m = re.match(r"[0-9a-f]+ <(\S+)>:$", line)
        if m:
            kernel = m.group(1)
            continue
        m = re.match(r"\s*v_(?:lshl|lshr|ashr)rev_[bi]64(?:_e64)? v\[\d+:\d+\], v(\d+),", line)
        if m:
            shifts += 1
            if int(m.group(1)) == last[kernel]:
                bad.append((kernel, line.strip()))
    return shifts, bad


def test_no_shift_by_the_last_register(tmp_path):
    g.load_library()   # (builds it if it is not there)
    tools = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "llvm", "bin")

    def run(tool, *args):
        return subprocess.run([os.path.join(tools, tool), *args], check=True, stdout=subprocess.PIPE, universal_newlines=True).stdout

    def look(item):
        path = str(tmp_path / ("%d.co" % item[0]))
        with open(path, "wb") as f:
            f.write(item[1])
        return _shifts(run("llvm-objdump", "-d", "--no-show-raw-insn", path), _last_registers(run("llvm-readelf", "--notes", path)))

    with concurrent.futures.ThreadPoolExecutor(4) as ex:
        found = list(ex.map(look, enumerate(_code_objects(build.LIB))))
    assert sum(shifts for shifts, _ in found) > 0
    bad = [x for _, b in found for x in b]
    assert not bad, "%d, the first: %s" % (len(bad), bad[0])


def test_a_shift_by_the_last_register_is_seen():
    notes = "    .symbol:         f.kd\n    .vgpr_count:     250\n    .symbol:         h.kd\n    .vgpr_count:     40\n"
    last = _last_registers(notes)
    assert last == {"f": 255, "h": 39}
    listing = "00 <f>:\n v_lshrrev_b64 v[2:3], v255, v[4:5]\n v_lshrrev_b64 v[2:3], v39, v[4:5]\n00 <h>:\n v_lshlrev_b64 v[2:3], v39, v[4:5]\n v_lshlrev_b64 v[2:3], 4, v[4:5]\n"
    shifts, bad = _shifts(listing, last)
    assert shifts == 3 and [k for k, _ in bad] == ["f", "h"]
