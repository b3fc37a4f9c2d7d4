"""What the library says that a call of the operators would run, without a GPU."""
import ctypes
import os
import subprocess

import pytest

import test_operators_forms_gpu as F
from paper_2112_15445_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE = 1, 2


def test_the_structure_and_the_names_match_the_header(tmp_path):
    fields = [f for f, _ in B.sc_launch_t._fields_]
    names = ["NOTHING", "NORM_LANES", "NORM_SAMPLE", "NORM_TWO", "ROWS", "TILE_64", "TILE_64_SPLIT", "TILE_128", "TILE_128_DEEP", "TILE_256"]
    src = tmp_path / "launch.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sparse_conv.h"\nint main(void) {printf("%zu\\n", sizeof(sc_launch_t));'
                   + "".join('printf("%%zu\\n", offsetof(sc_launch_t, %s));' % f for f in fields) + "".join('printf("%%d\\n", SC_FORM_%s);' % n for n in names) + "return 0; }\n")
    exe = tmp_path / "launch"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    c = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    assert c == [ctypes.sizeof(B.sc_launch_t)] + [getattr(B.sc_launch_t, f).offset for f in fields] + list(range(len(B.FORMS)))


@pytest.mark.parametrize("name,good,bad,nothing", [("GroupNorm", (1, 4, 32, 4), (1, 4, 32, 5), (0, 4, 32, 4)), ("BlockMatmul", (1, 16, 32), (1, 0, 32), (0, 16, 32)),
                                                   ("GroupedMatmul", (1, 16, 32, 2), (1, 16, 32, 0), (0, 16, 32, 2))])
def test_what_it_refuses(name, good, bad, nothing):
    good, bad, nothing = (getattr(B, name)(*sizes) for sizes in (good, bad, nothing))
    assert good.launch()["form"] != "nothing" and nothing.launch()["form"] == "nothing"
    with pytest.raises(B.SparseConvError) as e:
        bad.launch()
    assert e.value.status == SHAPE
    ask = getattr(B.lib(), good._name + "_launch")
    assert ask(None, ctypes.byref(B.sc_launch_t())) == NULL and ask(ctypes.byref(good.desc), None) == NULL


def test_the_group_norms_of_the_tests_reach_every_form():
    """The shapes that the GPU's tests of every form go through still select what they were taken for, and nothing is left out:
    each number of lanes and vectors of the one-launch forms, values and codes, x past the cache and through it."""
    seen = {False: set(), True: set()}
    for N, S, C, G, x_type, codes, kind, lanes, held, past in F.NORM_FORMS:
        l = B.GroupNorm(N, S, C, G, x_type=x_type, y_type="e4m3" if codes else x_type).launch()
        assert (l["form"], l["lanes"], l["held"], l["past_cache"]) == (kind, lanes, held, past)
        seen[codes].add((kind, lanes, held, past))
    lanes = {(256, 4), (512, 4), (512, 16), (1024, 16)}
    forms = {("norm two", 0, 0, 0)} | {("norm sample", t, u, 0) for t, u in ((256, 4), (1024, 4), (1024, 8))} | {("norm lanes", t, u, 0) for t, u in lanes}
    assert forms <= seen[True] and forms | {("norm lanes", t, u, 1) for t, u in lanes} <= seen[False]
    assert any(s[3] for s in seen[True])
    for table in (F.IN_PLACE, F.NOT_FINITE):
        assert {row[-1] for row in table} == {"norm lanes", "norm sample", "norm two"}


def test_the_products_of_the_tests_reach_every_form():
    F.test_the_shapes_of_the_tests_reach_every_form()
