"""Which form of the 4-bit product a call gets: the rule of launch_rows in
lcsm_q4.hip, evaluated from its source, so that tests can tell the forms that a
list of cases reaches."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_12982_amd", "csrc", "lcsm_q4.hip")


def _translate():
    with open(SOURCE) as f:
        text = f.read()
    body = re.search(r"hipError_t launch_rows\(const Q4Call& c, hipStream_t st\) \{\n(.*?)\n\}", text, re.S).group(1)
    out, depth = ["def pick(c_rows, c_N, c_K, SPG, size_E):", "    c_kb = (c_K + 127) // 128",
                  "    groups = lambda rt, nt: -(-tiles // nt) * -(-rows // rt)"], 1
    for line in re.sub(r"//.*", "", body).split("\n"):
        line = re.sub(r"\bc\.(\w+)", r"c_\1", line.strip()).replace("sizeof(E)", "size_E").replace("&&", "and")
        line = re.sub(r"return launch<E, SPG, (\w+), (\w+)>\(c, (\d+), st\);", r"return (\1, \2, \3)", line)
        pad = "    " * depth
        if not line or line.startswith("auto groups"):
            continue
        if line == "}":
            depth -= 1
        elif m := re.fullmatch(r"if \((.*)\) \{", line):
            out.append(f"{pad}if {m.group(1)}:")
            depth += 1
        elif m := re.fullmatch(r"if \((.*)\) (return .*)", line):
            out.append(f"{pad}if {m.group(1)}: {m.group(2)}")
        elif m := re.fullmatch(r"(?:constexpr int|const long long) (.*);", line):
            for name, value in (v.split(" = ", 1) for v in m.group(1).split(", ")):
                value = re.sub(r"^(.*) \? (\d+) : (\d+)$", r"\2 if \1 else \3", value).replace("/", "//")
                out.append(f"{pad}{name} = {value}")
        else:
            assert line.startswith("return "), line
            out.append(pad + line)
    space = {}
    exec("\n".join(out), space)
    return space["pick"]


_pick = _translate()


def form(R, N, K, group, size):
    """(bytes of a value, 32-input products a scale, row tiles, output tiles, waves at most)."""
    spg = {32: 1, 64: 2}.get(group, 4)
    return (size, spg) + _pick(R, N, K, spg, size)
