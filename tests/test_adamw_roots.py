"""The root of the AdamW step (csrc/adamw.cu, roots): one residual step from an approximate reciprocal root y of v,
    g = fl(v y),   r = fl(fl(v - g g) (y / 2) + g),
carried out here for every fp32 v of two binades and every y that the instruction's documented bound (PTX ISA, rsqrt.approx.ftz.f32: a
relative error of 2^-22.9 at most) allows.  Powers of four scale all of it exactly within 2^-100 .. 2^100: the residual is a multiple of
2^-46 of v's binade, no smaller than fp32's least number there.  CPU only."""
import numpy as np

# The v of [1, 4) for which some y within the bound gives another value than the correctly rounded root; tests/test_gpu_adamw.py takes
# these to the device.
SPECIAL = (1.9692776203155518, 3.7277493476867676)


def rounded_sum(a, b):
    """fp32 nearest to the exact a + b of fp64 arrays, |a| < |b|: the fp64 sum, its last bit odd where it is not exact."""
    hi = a + b
    lo = a - (hi - b)
    bits = hi.view(np.int64)
    bits = np.where((lo != 0) & ((lo < 0) == (hi > 0)), bits - 1, bits)        # towards zero
    return np.where(lo != 0, bits | 1, bits).view(np.float64).astype(np.float32)


def test_all_values_and_all_reciprocal_roots():
    found, step = set(), 1 << 21
    for first in range(0x3F800000, 0x40800000, step):
        v = np.arange(first, first + step, dtype=np.uint32).view(np.float32)
        exact, want = np.sqrt(v.astype(np.float64)), np.sqrt(v)
        near = (1 / exact).astype(np.float32)
        for off in range(-3, 4):
            y = (near.view(np.int32) + off).view(np.float32)
            allowed = np.abs(y.astype(np.float64) * exact - 1) <= 2.0 ** -22.9
            assert abs(off) < 3 or not allowed.any()                           # all that the bound allows are looked at
            if not allowed.any():
                continue
            g = (v * y).astype(np.float64)
            residual = (v.astype(np.float64) - g * g).astype(np.float32)       # exact in 64 bits, rounded once
            r = rounded_sum(residual.astype(np.float64) * (y.astype(np.float64) / 2), g)
            found.update(v[allowed & (r != want)].tolist())
    assert found == set(SPECIAL)
