"""Inline assembly of the kernel sources names every fixed register that it writes (no GPU)."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = sorted(glob.glob(os.path.join(ROOT, "paper_2606_28560_amd", "csrc", "*")))


def _statements(src):
    """(template, clobbers) of every asm statement."""
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", src):
        depth, i = 1, m.end()
        quoted = False
        while depth:
            c = src[i]
            if c == '"' and src[i - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            i += 1
        body = src[m.end():i - 1]
        parts, cur, quoted, depth = [], "", False, 0
        for a, c in enumerate(body):
            if c == '"' and body[a - 1] != "\\":
                quoted = not quoted
            if not quoted:
                depth += (c in "([") - (c in ")]")
                if c == ":" and depth == 0:
                    parts.append(cur)
                    cur = ""
                    continue
            cur += c
        parts.append(cur)
        yield "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', parts[0])), re.findall(r'"([^"]*)"', parts[3]) if len(parts) > 3 else []


def _written(template):
    """The fixed registers that the instructions of a template write: m0, vcc, exec, s<n>, v<n> as
    a first operand, and scc by scalar arithmetic."""
    out = set()
    for ins in re.split(r"\\n|\\t|;|\n", template):
        ins = ins.strip()
        if not ins:
            continue
        op, _, args = ins.partition(" ")
        first = args.split(",")[0].strip()
        if re.fullmatch(r"m0|vcc(_lo|_hi)?|exec(_lo|_hi)?|[sv]\d+|[sv]\[\d+:\d+\]", first):
            out.add(first)
        if re.match(r"s_(add|sub|addc|subb|and|or|xor|lshl|lshr|ashr|cmp|min|max|bfe|not|abs)", op):
            out.add("scc")
    return out


def test_fixed_registers_that_are_written_are_clobbers():
    seen = 0
    for path in SOURCES:
        for template, clobbers in _statements(open(path).read()):
            seen += 1
            assert _written(template) <= set(clobbers), (os.path.basename(path), template, clobbers)
    assert seen >= 5
    # the reader of the statements sees a missing one
    src = 'asm volatile("s_mov_b32 m0, %0\\n\\ts_add_u32 m0, m0, %1" : : "s"(a[0]), "s"(f(b)) : "memory", "scc");'
    (template, clobbers), = _statements(src)
    assert _written(template) == {"m0", "scc"} and clobbers == ["memory", "scc"]
