"""The order of the attention operators beside demotions and promotions, without a GPU (attention_order.cu): on the pool's compute
stream and on another one, with deferred packing, and inside a stream capture."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe, csrc = str(tmp_path_factory.mktemp("order") / "attention_order"), os.path.join(ROOT, "paper_2604_26968_b200", "csrc")
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a",
                    "-diag-suppress", "186", "--cudart", "none", "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", os.path.join(ROOT, "tests"),
                    os.path.join(csrc, "kvtier_host.cu"), os.path.join(csrc, "kv_attention_host.cu"),
                    os.path.join(ROOT, "tests", "attention_order.cu"), "-o", exe], check=True)
    return exe


def play(program, *args):
    r = subprocess.run([program, *map(str, args)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (args, r.stdout)


@pytest.mark.parametrize("gather", [0, 1 << 20])
@pytest.mark.parametrize("deferred", [0, 1])
def test_two_streams_beside_promotions(program, deferred, gather):
    for seed in range(40):
        play(program, seed, deferred, gather)


def test_captures(program):
    play(program, "capture")
