"""Host-side checks of the latent kernels' generated gfx950 code (no GPU needed): registers that go to memory, which wait
for the loads ahead when they come back, stay as few as they are; and what the compiler does not look after around the
direct loads into LDS, which are inline assembly."""
import os
import re
import shutil

import pytest

from paper_2607_05708_amd import build

pytestmark = pytest.mark.skipif(not (os.path.exists(build.HIPCC) or shutil.which("hipcc")),
                                reason="hipcc not available")

# Registers spilled and bytes of scratch a thread, by kernel; all others have none.  latent_attend_kernel<format, latent,
# rows / 32>, latent_expand_kernel<format, latent, head_dim>.
SPILLED = {"latent_attend_kernelILi0ELi512ELi4E": 38, "latent_attend_kernelILi1ELi512ELi4E": 27,
           "latent_attend_kernelILi2ELi512ELi4E": 11}
SCRATCH = {"latent_attend_kernelILi0ELi512ELi4E": 80, "latent_attend_kernelILi1ELi512ELi4E": 68,
           "latent_attend_kernelILi2ELi512ELi4E": 40, "latent_expand_kernelILi2ELi256ELi64E": 208,
           "latent_expand_kernelILi2ELi256ELi128E": 208}


@pytest.fixture(scope="module")
def asm():
    return {src: build.device_asm(src) for src in ("csrc/latent.hip", "csrc/latent_expand.hip")}


def test_registers_in_memory(asm):
    seen = set()
    for text in asm.values():
        kernels = re.findall(r"\.name:\s+(\S+)", text)
        spills, scratch = (re.findall(rf"\.{what}:\s+(\d+)", text)
                           for what in ("vgpr_spill_count", "private_segment_fixed_size"))
        assert len(kernels) == len(spills) == len(scratch) > 0
        for name, a, b in zip(kernels, spills, scratch):
            key = next((k for k in SCRATCH if k in name), None)
            seen.add(key)
            assert int(a) <= SPILLED.get(key, 0), f"{name}: {a} registers spilled"
            assert int(b) <= SCRATCH.get(key, 0), f"{name}: {b} bytes of scratch"
    assert seen >= set(SCRATCH)


def instructions(text):
    lines = (l.split(";")[0].strip() for l in text.splitlines())
    return [l for l in lines if l and not l.startswith(".") and not l.endswith(":")]


def test_direct_loads_wait_for_their_scalars(asm):
    # M0's write is followed by a wait state; a vector instruction that writes a scalar address stands 5 wait states before
    # the load at least (looked for in program order, in which blocks follow each other)
    code = instructions(asm["csrc/latent_expand.hip"])
    loads = 0
    for i, line in enumerate(code):
        m = re.match(r"global_load_lds_dwordx4 v\d+, s\[(\d+):(\d+)\]", line)
        if not m:
            continue
        loads += 1
        assert code[i - 1] == "s_nop 0" and code[i - 2].startswith("s_mov_b32 m0, "), code[i - 3:i + 1]
        states = 0
        for before in reversed(code[max(i - 8, 0):i]):
            w = re.match(r"v_(?:readfirstlane|readlane|cmp)\S* s\[?(\d+)(?::(\d+))?", before)
            if w and states < 5:
                wrote = range(int(w[1]), int(w[2] or w[1]) + 1)
                assert int(m[1]) not in wrote and int(m[2]) not in wrote, code[i - 8:i + 1]
            states += 1 + (int(before.split()[1]) if before.startswith("s_nop") else 0)
    assert loads
