"""Registers, LDS and spills of the attention over a cache in a microscaling format as built (the code objects' own metadata, no
GPU): the plan counts workgroups that a compute unit holds."""
import re

from test_kernel_registers import _kernels


def _waves(k):
    """Wavefronts of a SIMD that the registers allow: of 512, given out by eights."""
    return 512 // (-(-(k[".vgpr_count"]) // 8) * 8)


def test_few_rows():
    """Four wavefronts per workgroup; workgroups that the plan counts of a compute unit: three with one query tile, two with two or
    in 8 bits of 128.  Only of two tiles of heads of 64 in 4 bits one more would fit."""
    n = 0
    for name, k in _kernels().items():
        m = re.match(r"_ZN2ss13msa_mx_kernelILi(\d+)ELb([01])ELi(\d)E", name)
        if m:
            D, fp8, nt = int(m[1]), m[2] == "1", int(m[3])
            wgs = 3 if nt == 1 and not (fp8 and D == 128) else 2
            assert _waves(k) >= wgs and wgs * k[".group_segment_fixed_size"] <= 160 * 1024, name
            one_more = (wgs + 1) * k[".group_segment_fixed_size"] <= 160 * 1024 and _waves(k) > wgs
            assert one_more == (not fp8 and (D, nt) == (64, 2)), name
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
            n += 1
    assert n == 8


def test_shared_keys():
    """NW wavefronts of G groups; one workgroup per compute unit with one tile per wave, two with two tiles.  Two instances keep two
    and three values in scratch memory that are needed before and after the loop over the keys."""
    n, spills = 0, {}
    for name, k in _kernels().items():
        m = re.match(r"_ZN2ss18msa_mx_rows_kernelILi(\d+)ELb([01])ELi(\d)ELi(\d)ELi(\d)E", name)
        if m:
            D, fp8, nw, nt, g = (int(x) for x in m.groups())
            per_simd = -(-(nw * g * (2 if nt == 2 else 1)) // 4)
            assert _waves(k) >= per_simd, name
            if k[".vgpr_spill_count"]:
                spills[D, fp8, nw, nt, g] = k[".vgpr_spill_count"]
            n += 1
    assert n == 20
    assert set(spills) <= {(128, 1, 5, 1, 2), (64, 1, 5, 1, 3)} and all(v <= 3 for v in spills.values()), spills
