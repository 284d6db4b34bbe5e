"""The items of a plan or a release of pages, on the host, up to the largest sizes."""
import os
import subprocess

from paper_2607_17644_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_items_and_their_requests(tmp_path):
    exe = str(tmp_path / "page_items")
    r = subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I",
                        os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                        os.path.join(HERE, "host", "page_items.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
