"""The benchmark's traffic figures come from profiles that name the kernels' sources: those of the kernels that it times, and no others."""
import os
import shutil

import bench

CSRC = os.path.join("paper_2602_21477_amd", "csrc")


def copy(tmp_path, monkeypatch):
    os.makedirs(tmp_path / "paper_2602_21477_amd")
    shutil.copytree(os.path.join(bench.ROOT, CSRC), tmp_path / CSRC)
    shutil.copytree(os.path.join(bench.ROOT, "profiles"), tmp_path / "profiles")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path / CSRC


def test_other_operators_leave_the_figures(tmp_path, monkeypatch):
    csrc = copy(tmp_path, monkeypatch)
    was, traffic = bench.kernel_sources_sha(), bench.profiled_traffic("c4", "ip")
    (csrc / "pk_kv_more.hip").write_text("// another file of the key/value cache\n")
    with open(csrc / "pk_kv.hip", "a") as f:
        f.write("// a change\n")
    assert bench.kernel_sources_sha() == was and bench.profiled_traffic("c4", "ip") == traffic
    with open(csrc / "pk_scan.hip", "a") as f:
        f.write("// a change\n")
    assert bench.kernel_sources_sha() != was and bench.profiled_traffic("c4", "ip")[0] is None


def test_the_kernels_sources_need_nothing_of_the_cache():
    for name in os.listdir(os.path.join(bench.ROOT, CSRC)):
        if not name.startswith("pk_kv"):
            assert "pk_kv" not in open(os.path.join(bench.ROOT, CSRC, name)).read(), name
