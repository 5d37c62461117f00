"""Attention over the 4-bit cache for many rows: what its waves read of the first tile before they enter the loop over the tiles, the loop overwrites with the third, so a
barrier has to stand between.  A wave that lags is too rare for results to show that it is missing: looked for in the kernels as they are built, on every path."""
import re
import subprocess

import pytest

import paper_2407_11062_amd as eq
from test_kernel_registers import code_objects

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def kernels_of(listing):
    """{kernel: [(address, operation, branch target or None)]} of a disassembly"""
    out, name = {}, None
    for line in listing:
        m = re.match(r"([0-9a-f]+) <(.+)>:", line)
        if m:
            name, start = m[2], int(m[1], 16)
            out[name] = []
            continue
        m = re.match(r"\s+([a-z]\w+).*//\s*([0-9A-F]+):", line)
        if name and m:
            to = re.search(r"<[^<>]+\+0x([0-9a-f]+)>\s*$", line) if "branch" in m[1] else None
            out[name].append((int(m[2], 16), m[1], start + int(to[1], 16) if to else None))
    return out


def followers(code):
    at = {a: i for i, (a, _, _) in enumerate(code)}
    return [([at[to]] if to is not None else []) + ([i + 1] if op not in ("s_branch", "s_endpgm") and i + 1 < len(code) else []) for i, (_, op, to) in enumerate(code)]


def reached(starts, edges, stop=lambda i: False):
    seen, todo = set(), list(starts)
    while todo:
        i = todo.pop()
        if i not in seen:
            seen.add(i)
            if not stop(i):
                todo += edges[i]
    return seen


def unguarded(code):
    """the loop's writes to LDS that a path reaches from a read in front of the loop without a barrier; None without such a loop"""
    edges = followers(code)
    back = [[] for _ in code]
    for i, js in enumerate(edges):
        for j in js:
            back[j].append(i)
    barriers = [i for i, (_, op, _) in enumerate(code) if op == "s_barrier"]
    loops = [reached(edges[b], edges) & reached(back[b], back) for b in barriers]
    loops = [l for l in loops if any(code[i][1] == "ds_write_b128" for i in l)]
    if not loops:
        return None
    loop = max(loops, key=len)
    before = reached([j for i in loop for j in back[i]], back) - loop
    reads = [i for i in before if code[i][1] == "ds_read_b128"]
    assert reads
    hit = reached(reads, edges, stop=lambda i: code[i][1] == "s_barrier")
    return sorted(i for i in hit & loop if code[i][1] == "ds_write_b128")


def test_the_search_finds_what_it_is_for():
    text = ["0000000000000000 <k>:"] + [f"\t{op} // {4 * i:012X}: 00" + (f" <k+0x{to:x}>" if to is not None else "") for i, (op, to) in enumerate(
        [("ds_write_b128", None), ("s_barrier", None), ("s_cbranch_scc1", 0x24), ("ds_read_b128", None), ("s_nop", None),
         ("ds_read_b128", None), ("ds_write_b128", None), ("s_barrier", None), ("s_cbranch_scc0", 0x14), ("s_endpgm", None)])]
    assert unguarded(kernels_of(text)["k"]) == [6]
    text[5] = text[5].replace("s_nop", "s_barrier")
    assert unguarded(kernels_of(text)["k"]) == []


@pytest.fixture(scope="module")
def prompts(tmp_path_factory):
    out = {}
    for k, code in enumerate(code_objects(eq.LIB_PATH)):
        f = tmp_path_factory.mktemp("code") / f"{k}.co"
        f.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(f)], capture_output=True, text=True, check=True).stdout.splitlines()
        out.update({n: c for n, c in kernels_of(listing).items() if "k_kv_prompt" in n})
    return out


def test_the_loop_waits_for_the_reads_before_it(prompts):
    assert len(prompts) >= 20
    found = {n: unguarded(c) for n, c in prompts.items()}
    assert all(f is not None for f in found.values())
    assert not any(found.values()), {n: len(f) for n, f in found.items() if f}
