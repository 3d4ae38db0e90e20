"""The profile summaries and the digest that tells whether their figures belong to the tree's kernels."""
import os
import shutil
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2105_07829_amd", "csrc")
sys.path.insert(0, ROOT)
import bench  # noqa: E402

WORKLOADS = ["bert_large", "bert_base", "resnet50", "vgg16"]


@pytest.mark.parametrize("workload", WORKLOADS)
def test_a_profile_names_the_sources_of_its_kernels(workload):
    """The files on the SOURCES line hold, with what they include, every kernel of the first table."""
    total, digest, files = bench.recorded_traffic(workload, "W")
    assert total > 0 and len(digest) == 16 and int(digest, 16) >= 0 and files
    name = [n for n in os.listdir(os.path.join(ROOT, "profiles")) if n.startswith(f"bench_{workload}_")]
    assert len(name) == 1
    text = open(os.path.join(ROOT, "profiles", name[0])).read()
    assert text.count("SOURCES ") == 1
    sources = "".join(open(os.path.join(CSRC, f)).read() for f in [*files, "cluster_launch.hpp"])
    kernels = {w.split("<")[0].split("::")[1] for w in text.split() if w.startswith("bpc::")}
    kernels |= {w.split("<")[1].split("::")[1] for w in text.split() if w.startswith("bpc::cluster_kernel<bpc::")}
    assert len(kernels) > 4
    for k in kernels:
        assert f" {k}(" in sources or f"struct {k} " in sources, k


@pytest.mark.parametrize("workload", WORKLOADS)
def test_the_digest_follows_the_files_a_workload_is_compiled_from(workload, tmp_path):
    _, _, files = bench.recorded_traffic(workload, "W")
    csrc = shutil.copytree(CSRC, tmp_path / "csrc")
    before, whole = bench.sources_digest(files, csrc), bench.sources_digest(None, csrc)
    assert before == bench.sources_digest(files)

    def changed(name):
        with open(csrc / name, "a") as f:
            f.write("// x\n")
        return bench.sources_digest(files, csrc) != before
    for name in ("logits_topk.hip", "distill_student.hpp", "distill_call.hpp", "distill_geometry.hpp", "probe.hip"):
        assert not changed(name), name
    assert bench.sources_digest(None, csrc) != whole
    for name in (*files, "device_utils.hpp", "geometry.hpp", "kernels.hpp", "sources.hpp"):
        shutil.rmtree(csrc)
        shutil.copytree(CSRC, csrc)
        assert changed(name), name


def test_no_profile_no_traffic():
    assert bench.recorded_traffic("no such workload", "W") == (None, None, None)
