"""Kernels that are launched to overlap their predecessor wait for it on every way out: what is launched behind them relies on
their end to mean that everything earlier has ended too.  Read from the sources; no GPU."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_22737_b200", "csrc")


def _source():
    text = "\n".join(open(p).read() for p in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))))
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def _launched_behind(text):
    """Names of the kernels that launch_behind is given, directly or as a pointer chosen beforehand."""
    names = set()
    for call in re.finditer(r"launch_behind\(\s*([^,]+?)\s*,", text):
        names |= set(re.findall(r"\w+_kernel", call.group(1)))
        if call.group(1) == "kern":
            names |= set(re.findall(r"\w+_kernel", re.findall(r"auto kern = ([^;]+);", text[:call.start()])[-1]))
    return sorted(names)


def _body(text, name):
    m = re.search(r"__global__[^;{}]*?\b" + name + r"\s*\([^{;]*\)\s*\{", text)
    depth, at = 1, m.end()
    while depth:
        depth += {"{": 1, "}": -1}.get(text[at], 0)
        at += 1
    return text[m.end():at]


def test_the_kernels_are_found():
    assert {"attn_shared_kernel", "conf_adjusted_kernel", "conf_commit_kernel", "rope_stage_kernel", "shared_merge_kernel",
            "shared_plan_kernel", "shared_plan_small_kernel"} <= set(_launched_behind(_source()))


@pytest.mark.parametrize("name", _launched_behind(_source()))
def test_no_way_out_without_the_wait(name):
    body = _body(_source(), name)
    if "WaitAtExit" in body:                    # an object whose destructor waits, made before anything can return
        assert body.index("WaitAtExit") < (body.index("return;") if "return;" in body else len(body))
        return
    assert "grid_dependency_wait();" in body
    for m in re.finditer(r"\breturn;", body):
        assert "grid_dependency_wait();" in body[:m.start()], body[:m.end()][-200:]
