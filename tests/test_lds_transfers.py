"""Transfers from memory straight into LDS, in the code objects of liblcsm.so
(host only).  The compiler does not wait for such a transfer where LDS is read:
the kernel has to, and a wait that is missing shows in no result while the
transfer happens to be the faster one.  In the kernels that hold one stage of
operands in LDS nothing may be read from it while a transfer is on its way."""
import re
import shutil
import subprocess

import pytest

from test_kernel_resources import LIB, READELF, _code_objects

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# Loads and stores of memory, which vmcnt counts in the order of their issue.
MEMORY = re.compile(r"(buffer|global|scratch|flat)_(load|store|atomic)")
LINE = re.compile(r"\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+):")
TARGET = re.compile(r"<[^>]*?(?:\+0x([0-9a-f]+))?>\s*$")


@pytest.fixture(scope="module")
def chunk_kernels(tmp_path_factory):
    """(address, opcode, operands, branch target) lists of every k_ssm_chunks by mangled name."""
    if not (shutil.which(OBJDUMP) and shutil.which(READELF)):
        pytest.skip("llvm-objdump or llvm-readelf is not installed")
    d = tmp_path_factory.mktemp("co")
    with open(LIB, "rb") as f:
        blob = f.read()
    out = {}
    for k, co in enumerate(_code_objects(blob)):
        if b"k_ssm_chunks" not in co:
            continue
        path = d / f"{k}.co"
        path.write_bytes(co)
        symbols = subprocess.run([READELF, "-sW", str(path)], check=True, capture_output=True, text=True).stdout
        names = sorted({w for w in symbols.split() if "k_ssm_chunks" in w and not w.endswith(".kd")})
        text = subprocess.run([OBJDUMP, "-d", "--disassemble-symbols=" + ",".join(names), str(path)], check=True,
                              capture_output=True, text=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\S+)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", text, re.S | re.M):
            code = []
            for line in body.split("\n"):
                m = LINE.match(line)
                if m:
                    code.append([int(m.group(3), 16), m.group(1), m.group(2), None])
                    if m.group(1).startswith(("s_branch", "s_cbranch")):
                        code[-1][3] = code[0][0] + int(TARGET.search(line).group(1) or "0", 16)
            out[name] = code
    assert out
    return out


def early_reads(code):
    """Addresses of the LDS reads that a path reaches with a transfer into LDS on
    its way.  Along a path the state is how many memory instructions have been
    issued from the newest transfer on (the fewest, where paths meet): a wait that
    leaves fewer than that has waited for it."""
    index = {c[0]: i for i, c in enumerate(code)}
    state, found, todo = {0: 0}, set(), [0]
    while todo:
        i = todo.pop()
        since = state[i]
        at, op, args, target = code[i]
        if MEMORY.match(op):
            if re.search(r"\blds\b", args):
                since = 1
            elif since:
                since += 1
        elif op == "s_waitcnt":
            m = re.search(r"vmcnt\((\d+)\)", args)
            if m and int(m.group(1)) < since:
                since = 0
        elif op.startswith("ds_read") and since:
            found.add(at)
        nxt = [index[target]] if target is not None else []
        if op not in ("s_branch", "s_endpgm", "s_setpc_b64"):
            nxt.append(i + 1)
        for n in nxt:
            old = state.get(n)
            new = since if old is None else since if not old else old if not since else min(old, since)
            if old is None or new != old:
                state[n] = new
                todo.append(n)
    return found


def test_the_walk_finds_a_missing_wait():
    """The walk itself, on code made here: a wait that leaves the transfer on its
    way, one that does not, and a way around it."""
    load, copy = (1, "buffer_load_dword", "v1, v2, s[0:3], 0 offen", None), (0, "buffer_load_dwordx4", "v1, s[0:3], 0 offen lds", None)
    read, end = "ds_read_b128", "s_endpgm"
    at = lambda ops: [[k, *o[1:]] for k, o in enumerate(ops)]  # noqa: E731
    assert early_reads(at([copy, load, (0, "s_waitcnt", "vmcnt(0)", None), (0, read, "", None), (0, end, "", None)])) == set()
    assert early_reads(at([copy, load, (0, "s_waitcnt", "vmcnt(1)", None), (0, read, "", None), (0, end, "", None)])) == set()
    assert early_reads(at([load, copy, (0, "s_waitcnt", "vmcnt(1)", None), (0, read, "", None), (0, end, "", None)])) == {3}
    around = [copy, (0, "s_cbranch_scc1", "", 3), (0, "s_waitcnt", "vmcnt(0) lgkmcnt(0)", None), (0, read, "", None),
              (0, end, "", None)]
    assert early_reads(at(around)) == {3}


@pytest.mark.parametrize("blocks", [1, 2])
@pytest.mark.parametrize("out", [0, 1])
def test_one_stage_is_read_after_it_has_arrived(chunk_kernels, blocks, out):
    """k_ssm_chunks<E, blocks, out, PAIR> of up to 64 states, for three types and both alignments."""
    mine = {n: c for n, c in chunk_kernels.items() if re.search(rf"Li{blocks}ELb{out}ELb[01]E", n)}
    assert len(mine) == 6
    for name, code in mine.items():
        assert any("lds" in c[2] for c in code) and any(c[1].startswith("ds_read") for c in code)
        assert early_reads(code) == set(), name
