"""Bounds of kv_attend that do not fit its launches, refused by the host side without a GPU (attention_limits.cu)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_bounds_that_fit_and_others(tmp_path):
    exe, csrc = str(tmp_path / "limits"), os.path.join(ROOT, "paper_2604_26968_b200", "csrc")
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a",
                    "-diag-suppress", "186", "--cudart", "none", "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", os.path.join(ROOT, "tests"),
                    os.path.join(csrc, "kvtier_host.cu"), os.path.join(csrc, "kv_attention_host.cu"),
                    os.path.join(ROOT, "tests", "attention_limits.cu"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, "\n".join(sorted(set((r.stdout + r.stderr).splitlines())))
