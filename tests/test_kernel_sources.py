"""Rules of the kernels that no run can show to be kept, read from their sources."""
import os
import re

from paper_2407_00952_b200 import build


def sources():
    for name in sorted(os.listdir(build.CSRC)):
        if name.endswith((".cu", ".cuh")):
            with open(os.path.join(build.CSRC, name)) as f:
                yield name, re.sub(r"//[^\n]*", "", f.read())


def test_every_bounded_wait_is_looked_at():
    """A wait that ran out returns false: the data is not there, and a kernel that goes on computes with what lay in its place."""
    waits = 0
    for name, text in sources():
        waits += len(re.findall(r"\bmbar_wait(?:_warp)?\(", text))
        ignored = re.findall(r"(?<=[;{})])\s*((?:tc::)?mbar_wait(?:_warp)?\([^;]*;)", text)
        assert not ignored, (name, ignored)
    assert waits > 20


# Kernels of calls that allow an output to be an input: the parameters that may point at the same memory.
MAY_ALIAS = {"rmsnorm_quantize_kernel": ("x", "resid", "h"), "rmsnorm_bwd_kernel": ("dy", "resid", "dx"), "distill_kernel": ("logits", "grad"),
             "distill_ring_kernel": ("logits", "grad"), "distill_warp_kernel": ("logits", "grad")}


def test_what_may_alias_is_not_promised_apart():
    """Writing through one __restrict__ pointer what another reads is undefined: a compiler may read an input again after the output lies
    over it, whatever today's does."""
    seen = set()
    for name, text in sources():
        for kernel, params in MAY_ALIAS.items():
            for m in re.finditer(r"__global__[^;{]*?\b" + kernel + r"\(([^)]*)\)\s*\{", text):
                seen.add(kernel)
                declared = [p.split() for p in m.group(1).split(",")]
                for p in params:
                    mine = [d for d in declared if d[-1] == p]
                    assert len(mine) == 1 and "__restrict__" not in mine[0], (name, kernel, p)
    assert seen == set(MAY_ALIAS)
