"""What the compiler gives the kernels of the norm, the recurrence and the distillation loss (on the CPU): no packed fp32 arithmetic,
and registers as the comments beside them count on them."""
import re
import shutil

import pytest

from paper_2004_14020_amd import build
from test_layer_kernels import compiled                       # noqa: F401  (a fixture)

pytestmark = [pytest.mark.skipif(shutil.which(build.hipcc()) is None, reason="hipcc not available"),
              pytest.mark.parametrize("compiled", ["norm", "recurrence", "distillation"], indirect=True, scope="module")]


def test_no_packed_fp32_arithmetic(compiled):                 # noqa: F811
    asm, kernels = compiled
    assert len(kernels) > 3 and "s_endpgm" in asm
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm)


def test_registers(compiled):                                 # noqa: F811
    asm, kernels = compiled
    for name, r in kernels.items():
        if re.search(r"k_norm_gradient<(true, 4|false, 8), 16>", name):
            # rows of more than 16384 columns: the sums of the gain gradient do not fit beside the row, and wait in memory
            assert r["ScratchSize [bytes/lane]"] <= 256, (name, r)
        else:
            assert r["VGPRs Spill"] == 0 and r["ScratchSize [bytes/lane]"] == 0, (name, r)


def test_wavefronts(compiled):                                # noqa: F811
    """Of the kernels that are bound by memory, as many to a SIMD as their figures were measured with."""
    asm, kernels = compiled
    least = {r"k_norm<.*, [124], \d+>": 8, r"k_walk_maps": 8, r"k_walk_tokens<true, 2, true": 5, r"k_walk_tokens<false, 2, true": 4,
             r"k_walk_tokens<\w+, \d, false": 6, r"k_distillation<.*, 0, \d+, 32, 0>": 8, r"k_distillation<": 4}
    for name, r in kernels.items():
        for pattern, waves in least.items():
            if re.search(pattern, name):
                assert r["Occupancy [waves/SIMD]"] >= waves, (name, r)
                break
