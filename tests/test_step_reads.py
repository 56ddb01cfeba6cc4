"""What the verification reads of arrays that it is promised not to need whole, on the host (CPU only): step_reads.cpp runs the kernels' own
functions before pages that no one may read."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_nothing_is_read_that_need_not_be_there(tmp_path):
    """The number behind the last row's, and the draft model's logits of a greedy sequence.  (Without optimization, so that every load that
    is written is made.)"""
    out = str(tmp_path / "step_reads")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O0", "-std=c++17", "-Wno-everything", "-x", "hip", "--cuda-host-only",
                    "-I", os.path.join(ROOT, "paper_2507_01663_amd", "csrc"), "-o", out, os.path.join(ROOT, "tests", "step_reads.cpp")], check=True, timeout=300)
    r = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.split() == ["numbers", "greedy", "drafts"], (r.returncode, r.stdout)
