"""Set-up of the 8-bit operators' kernels: one function does it, behind a lock.

It writes what launches on other threads read (how many clusters run at a time, a driver entry point), so no path may write it again
while a product is being launched.  Read from the sources: nothing runs on a GPU."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_16843_b200", "csrc")


def code(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


def functions(text):
    """(name, body) of each function that starts at the left margin."""
    for m in re.finditer(r"^(?:template <[^\n]*>\n)?[\w:*<>, ]*?(\w+)\([^;{}]*\) \{\n(.*?)^\}", text, re.M | re.S):
        yield m.group(1), m.group(2)


def callers(name):
    return {(os.path.basename(p), f) for p in glob.glob(os.path.join(CSRC, "*.cu")) for f, body in functions(code(p))
            if re.search(r"\b%s\(" % name, body)}


@pytest.mark.parametrize("name,caller", [("setup_dense8_tc", ("dense8_api.cu", "ready")), ("setup_dense8_split", ("dense8_tc.cu", "setup_dense8_tc"))])
def test_only_the_locked_function_sets_up(name, caller):
    assert callers(name) == {caller}


def test_the_function_holds_its_lock():
    body = dict(functions(code(os.path.join(CSRC, "dense8_api.cu"))))["ready"]
    assert 0 <= body.find("lock_guard") < body.find("d.ready") < body.find("setup_dense8_tc")


def test_all_public_entries_pass_through_it():
    bodies = dict(functions(code(os.path.join(CSRC, "dense8_api.cu"))))
    for entry in ("llmcache_norm", "llmcache_dense", "setup_eight"):
        assert "ready(&dev, &d)" in bodies[entry]
    assert "setup_eight()" in dict(functions(code(os.path.join(CSRC, "layer_api.cu"))))["llmcache_layer_quantise"]


def test_driver_entry_points_are_looked_up_behind_a_lock():
    body = dict(functions(code(os.path.join(CSRC, "tensor_map.cu"))))["tensor_map_setup"]
    assert 0 <= body.find("lock_guard") < body.find("g_encode")


@pytest.mark.parametrize("name", ["setup_norm", "setup_dense8_few"])
def test_norm_and_few_rows_are_set_up_with_the_others(name):
    assert callers(name) == {("dense8_api.cu", "ready")}


def test_nothing_is_set_up_by_a_launch():
    for file in ("norm.cu", "dense8_tc.cu", "dense8_split.cu", "dense8_few.cu"):
        for f, body in functions(code(os.path.join(CSRC, file))):
            if "cudaFuncSetAttribute" in body or "cudaOccupancyMax" in body:
                assert f.startswith("setup_"), (file, f)
    assert "setup_eight()" in dict(functions(code(os.path.join(CSRC, "layer_api.cu"))))["llmcache_layer_rms"]
