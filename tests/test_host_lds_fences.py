"""Values that lanes of a wave hand each other through LDS, in the sources: __builtin_amdgcn_wave_barrier() orders no memory accesses, so that a lane that did not write may
legally go on with what it read before; fences of the wave around it do (they are no instructions)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2308_10087_amd", "csrc")


def test_wave_barriers_of_the_answers_stand_between_fences():
    lines = [l for l in open(os.path.join(CSRC, "logprobs.hip")).read().splitlines() if re.search(r"__builtin_amdgcn_\w+\(", l)]
    at = [i for i, l in enumerate(lines) if "wave_barrier" in l]
    assert at
    for i in at:
        assert '__builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront")' in lines[i - 1], lines[i - 1:i + 2]
        assert '__builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront")' in lines[i + 1], lines[i - 1:i + 2]
