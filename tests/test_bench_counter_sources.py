"""Which sources the committed counters of the GEMM kernels depend on: the
operators' files are none of them."""
import os
import re
import shutil

import bench

PACKAGE = "paper_2608_18469_amd"
OPERATORS = ("csrc/ops.hip", "csrc/ops.h", "csrc/ops_api.cpp")


def test_operator_sources_leave_the_counters_valid(tmp_path, monkeypatch):
    shutil.copytree(os.path.join(bench.ROOT, PACKAGE, "csrc"), tmp_path / PACKAGE / "csrc")
    shutil.copy(os.path.join(bench.ROOT, PACKAGE, "build.py"), tmp_path / PACKAGE)
    want = bench.kernel_source_hash(), bench.kernel_source_hash(bench.TF_SOURCES)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))

    def changed(name):
        path = tmp_path / PACKAGE / name
        old = path.read_text()
        path.write_text(old + "\n// another line\n")
        got = bench.kernel_source_hash(), bench.kernel_source_hash(bench.TF_SOURCES)
        path.write_text(old)
        return got

    for name in OPERATORS:
        assert changed(name) == want, name
    for name in ("csrc/kernels.hip", "csrc/internal.h", "build.py"):
        assert all(a != b for a, b in zip(changed(name), want)), name
    assert changed("csrc/tf_api.cpp")[0] == want[0] and changed("csrc/tf_api.cpp")[1] != want[1]


def test_operators_are_declared_in_a_header_of_their_own():
    with open(os.path.join(bench.ROOT, PACKAGE, "csrc", "ops.h")) as f:
        names = re.findall(r"^struct (\w+)", f.read(), re.M)
    assert {"RopeArgs", "NormArgs", "NormBwdArgs", "DropArgs"} <= set(names)
    with open(os.path.join(bench.ROOT, PACKAGE, "csrc", "internal.h")) as f:
        text = f.read()
    assert not any(re.search(rf"\b{n}\b", text) for n in names)
