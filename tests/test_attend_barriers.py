"""Attention's waves join their results through the LDS that their next item's keys and values go to.  So in the
machine code no way leads from the barrier in front of the join to a write into LDS but through another barrier: the
waves that have no rows to join, or are through with theirs, would write over what others still read."""
import importlib.util
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_14636_amd", "csrc")


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    spec = importlib.util.spec_from_file_location("stride_build", os.path.join(CSRC, "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    out = str(tmp_path_factory.mktemp("asm") / "attend.s")
    subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(CSRC, "attend.hip"), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        return f.read()


def flow(body):
    """Instructions of a kernel, and the instructions that may follow each."""
    code, label = [], {}
    for line in body.split("\n"):
        line = line.split(";")[0].strip()
        if m := re.match(r"(\.L\w+):", line):
            label[m.group(1)] = len(code)
        elif line and not line.startswith("."):
            code.append(line)
    after = []
    for i, x in enumerate(code):
        op = x.split()[0]
        assert op not in ("s_setpc_b64", "s_swappc_b64"), x
        to = [] if op in ("s_endpgm", "s_branch") else [i + 1]
        if op.startswith(("s_branch", "s_cbranch")):
            to.append(label[x.split()[1]])
        after.append(to)
    return code, after


def reached(after, start, stop):
    """Instructions on the ways from behind `start` up to (and with) those in `stop`."""
    seen, todo = set(), list(after[start])
    while todo:
        i = todo.pop()
        if i not in seen:
            seen.add(i)
            if i not in stop:
                todo += after[i]
    return seen


def test_the_join_is_read_before_lds_is_written(assembly):
    names = re.findall(r"^(\S*13attend_kernel\S*):", assembly, re.M)
    assert len(names) >= 10
    for name in names:
        code, after = flow(assembly.split(f"\n{name}:", 1)[1].split(".Lfunc_end", 1)[0])
        barrier = {i for i, x in enumerate(code) if x.startswith("s_barrier")}
        # results: the stores of the loop over items (the plan's own are in front of it)
        store = {i for i, x in enumerate(code) if x.startswith("global_store") and i in reached(after, i, ())}
        write = {i for i, x in enumerate(code) if x.startswith("ds_write") or x.endswith(" lds") or "load_lds" in x}
        joins = 0
        for b in barrier:
            seen = reached(after, b, barrier)
            if seen & store:
                joins += 1
                assert not seen & write, (name, [code[i] for i in sorted(seen & write)][:3])
        assert joins and store and write, name
