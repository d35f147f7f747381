"""The kernels of the 8-bit projections and the 4-bit cache, compiled to assembly with the library's flags (no GPU needed): none spills,
none uses packed fp32, and the largest products' main loop, whose copies into LDS and waits are placed by hand, holds what its waits count
on: a meeting of the waves, the copies of one step, the reads of one step and its products, and no other memory instruction."""
import re

import pytest

from test_kernel_codegen import _assembly


def _kernels(lines):
    """name -> (body, descriptor) of every kernel"""
    out = {}
    for i, l in enumerate(lines):
        m = re.match(r"^\t\.amdhsa_kernel (\S+)", l)
        if m:
            start = next(j for j in range(i, -1, -1) if lines[j].startswith(m.group(1) + ":"))
            out[m.group(1)] = (lines[start:i], lines[i:i + 80])
    return out


@pytest.mark.parametrize("source,least", [("koala_int8", 35), ("koala_paged", 20)])
def test_no_kernel_spills_or_uses_packed_fp32(source, least):
    kernels = _kernels(_assembly(source))
    assert len(kernels) >= least
    for name, (body, desc) in kernels.items():
        scratch = next(int(l.split()[-1]) for l in desc if ".amdhsa_private_segment_fixed_size" in l)
        assert scratch == 0 and not any("scratch_" in l for l in body), f"{name} spills"
        assert not any(re.search(r"\bv_pk_(add|mul|fma)_f32\b", l) for l in body), f"{name} uses packed fp32"


@pytest.mark.parametrize("tm", [5, 6, 7, 8])
def test_the_largest_products_main_loop_holds_what_its_waits_count_on(tm):
    body, _ = next(k for n, k in _kernels(_assembly("koala_int8")).items() if f"k_linear_wideILi{tm}E" in n)
    code = [re.sub(r"\s+", " ", l.split("//")[0].strip()) for l in body]
    code = [l for l in code if l and l[0] not in ";." and not l.endswith(":")]
    meets = [i for i, l in enumerate(code) if l == "s_waitcnt vmcnt(8) lgkmcnt(0)" and code[i + 1] == "s_barrier"]
    assert len(meets) == 3                       # before the first read, and two a turn of the loop
    end = next(i for i, l in enumerate(code) if i > meets[2] and l == "s_waitcnt vmcnt(0) lgkmcnt(0)")
    copies = [i for i, l in enumerate(code) if l.endswith("offen lds")]
    assert len([i for i in copies if i < meets[0]]) == 12          # three steps ahead
    loop = code[meets[0]:end]                    # a step read and one copied before the turns, then two steps a turn, two products' worth
    memory = [l for l in loop if re.match(r"(buffer|global|flat|scratch)_", l)]
    assert len(memory) == 12 and all(l.startswith("buffer_load_dwordx4") and l.endswith("lds") for l in memory), memory
    assert sum(l.startswith("ds_read_b128") for l in loop) == 3 * (tm + 4)
    assert sum(l.startswith("v_mfma_i32_16x16x64_i8") for l in loop) == 2 * 4 * tm
    assert not any(re.match(r"ds_(write|bpermute|swizzle)|s_(load|buffer_load)|v_(readlane|readfirstlane)", l) for l in code[meets[0]:copies[-1]])
    for i in copies:                             # a copy's place in LDS is set right before it
        assert code[i - 2].startswith("s_mov_b32 m0,") and code[i - 1] == "s_nop 4"
