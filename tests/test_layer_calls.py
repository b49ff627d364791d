"""How the calls that fill gradient tensors check their arguments: what that costs, and which memory may lie where.  No GPU call is
made."""
import os
import random
import shutil
import subprocess

import pytest

import paper_2004_14020_amd as cm
from paper_2004_14020_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2004_14020_amd", "csrc")


def test_calls_allocate_nothing(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    exe, libdir = str(tmp_path / "alloc_check"), os.path.dirname(binding.LIB_PATH)
    subprocess.run(["gcc", "-std=gnu99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "host", "alloc_check.c"), "-L", libdir, "-l:libcaramel.so",
                    "-Wl,-rpath," + libdir, "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "alloc_check ok" in res.stdout, res.stdout + res.stderr


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_overlap_of_buffers_and_interleaved_rows(tmp_path):
    exe = str(tmp_path / "memory_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    os.path.join(ROOT, "tests", "host", "memory_check.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "memory_check ok" in res.stdout, res.stdout[-2000:] + res.stderr[-2000:]


def test_rows_that_interleave_by_less_than_their_length_are_refused():
    """Two workers in one array, the second one column too early or too late."""
    a, width = 1 << 20, 16
    plan = cm.Plan(2, [64])
    for second in (width - 1, width + 1):
        at = [a, a + 4 * second]
        for call in (lambda: plan.embedding_lookup([5 * a] * 2, 8, width, [6 * a] * 2, [5, 5], at, out_pitch=2 * width),
                     lambda: plan.checkpoint_load([5 * a, 6 * a], [5, 5], width, at, pitch=2 * width)):
            with pytest.raises(cm.CaramelError) as e:
                call()
            assert e.value.status == binding.EINVAL and "overlap" in str(e.value)
    plan.close()


def test_a_workspace_serves_fewer_tokens():
    """Also at the steps from short chunks of the sorted tokens to longer ones, and between the weight gradient's kernels."""
    rng = random.Random(3)
    for _ in range(300):
        world, k, outputs = rng.choice([1, 2, 3, 8, 16, 64]), int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 11))
        plan = cm.Plan(world, [k * outputs])
        steps = [16384 // world + d for d in (-9, -1, 0, 1, 9)] + [32 * k + d for d in (-17, -1, 0, 1)]
        tokens = sorted(max(0, t) for t in steps + [int(2 ** rng.uniform(0, 18)) for _ in range(20)])
        for size in (lambda n: plan.embedding_workspace(0, outputs, [n] * world),
                     lambda n: plan.weight_gradient_workspace(0, k, [n] * world)):
            sizes = [size(n) for n in tokens]
            assert sizes == sorted(sizes), (world, k, outputs, tokens, sizes)
        plan.close()
