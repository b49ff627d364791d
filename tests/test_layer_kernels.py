"""What the compiler gives the kernels that fill gradient tensors (on the CPU): no packed fp32 arithmetic, and
registers as the comments beside the kernels count on them."""
import re
import shutil
import subprocess

import pytest

from paper_2004_14020_amd import build

pytestmark = pytest.mark.skipif(shutil.which(build.hipcc()) is None, reason="hipcc not available")


@pytest.fixture(scope="module", params=["embedding", "checkpoint", "weight_gradient"])
def compiled(request):
    """(assembly, {kernel: {quantity: value}})"""
    res = subprocess.run([build.hipcc(), *build.flags(), "--cuda-device-only", "-S", f"{build.HERE}/csrc/{request.param}.hip",
                          "-o", "-", "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-2000:]
    reports = res.stderr.split("Function Name: ")[1:]
    names = subprocess.run(["c++filt"], input="\n".join(r.split()[0] for r in reports), capture_output=True, text=True,
                           check=True).stdout.splitlines()
    return res.stdout, {n: {k.strip(): int(v) for k, v in re.findall(r"remark: [^\n]*?  +([A-Z][^:\n]*): (\d+)", r)}
                        for n, r in zip(names, reports)}


def test_no_packed_fp32_arithmetic(compiled):
    asm, kernels = compiled
    assert len(kernels) > 3 and "s_endpgm" in asm
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm)


def test_registers(compiled):
    asm, kernels = compiled
    for name, r in kernels.items():
        if "k_weight_gradient<8" in name or "k_weight_gradient_short" in name:
            # two wavefronts per SIMD; what does not fit goes to memory before and after the loop over the tokens
            assert r["Occupancy [waves/SIMD]"] >= 2 and r["ScratchSize [bytes/lane]"] <= 160, (name, r)
        else:
            assert r["VGPRs Spill"] == 0 and r["ScratchSize [bytes/lane]"] == 0, (name, r)


def test_the_loop_over_the_tokens_keeps_to_registers(compiled):
    """Between two products of a loop, no scratch access."""
    asm, kernels = compiled
    bodies = re.findall(r"^(_ZN\S*k_weight_gradientI\S*):.*?s_endpgm", asm, re.S | re.M)
    for m in re.finditer(r"^(_ZN\S*k_weight_gradientI\S*):[^\n]*\n(.*?)s_endpgm", asm, re.S | re.M):
        loops = re.findall(r"^(\.LBB\S+):[^\n]*Inner Loop Header[^\n]*\n(.*?)s_cbranch_\w+ \1\b", m.group(2), re.S | re.M)
        walks = [body for _, body in loops if "mfma" in body]
        assert len(walks) == 2, m.group(1)                   # with and without the sums for the bias
        assert all("scratch_" not in body for body in walks), m.group(1)
    assert bool(bodies) == any("k_weight_gradient<" in n for n in kernels)
