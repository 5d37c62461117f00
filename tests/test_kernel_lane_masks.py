"""Registers that the compiler parks in accumulation registers or scratch while some lanes are off.  It has put such a copy between the restoring of an inner and of an outer
mask of lanes, where the lanes that skipped the branch lost the value (the streamed attention with heads of 256 in groups of 32, when a look-up in the page table was a branch
in a branch).  Looked for in the kernels as they are built: no copy stands between two restores of the mask."""
import re
import subprocess

import paper_2407_11062_amd as eq
from test_kernel_registers import code_objects

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def parked(listing):
    """(kernel, copies) that stand between two restores of exec with no branch between them"""
    found, kernel, copies = [], None, None
    for line in listing:
        m = re.match(r"[0-9a-f]+ <(.+)>:", line)
        text = line.split("//")[0].strip()
        if m:
            kernel, copies = m[1], None
        elif text.startswith("s_or_b64 exec, exec,"):
            if copies:
                found.append((kernel, copies))
            copies = []
        elif "branch" in text or "endpgm" in text or re.match(r"s_\w*saveexec", text) or re.match(r"s_mov_b64 exec", text):
            copies = None
        elif copies is not None and text.startswith(("v_accvgpr_write", "scratch_store")):
            copies.append(text)
    return found


def test_the_search_finds_what_it_is_for():
    listing = ["0000 <k>:", " s_and_saveexec_b64 s[8:9], vcc // x", " s_cbranch_execz 9 // x", " s_and_saveexec_b64 s[12:13], vcc // x", " v_add_u32 v1, v2, v3 // x",
               " s_or_b64 exec, exec, s[12:13] // x", " v_accvgpr_write_b32 a158, v104 // x", " s_mov_b32 s33, s76 // x", " s_or_b64 exec, exec, s[8:9] // x"]
    assert parked(listing) == [("k", ["v_accvgpr_write_b32 a158, v104"])]
    listing[6], listing[8] = listing[8], listing[6]
    assert parked(listing) == []


def test_no_copy_between_two_restores(tmp_path):
    found = []
    for k, code in enumerate(code_objects(eq.LIB_PATH)):
        f = tmp_path / f"{k}.co"
        f.write_bytes(code)
        found += parked(subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(f)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert found == []
