"""The norm into eight bits where its results lie below the normal 32-bit numbers, shared by the CPU checker's tests and the device's (test helper, not collected)."""
import numpy as np

import plain_cases as pc
import plain_rows_cases as rc


def check_norm_mx(b, dtype, rows, n, power):
    """Results around 2^power: below 2^-127 the blocks' scale is the least and the codes' step 2^-136, of which 32 bits hold 2^13 parts; below 2^-149 nothing else than whether it is 0 is left."""
    rng = np.random.default_rng([rows, n, -power, 41])
    x = b.make(pc.normal(rng, rows, n), dtype)
    w = b.make(np.exp2(power + rng.uniform(-2, 2, size=n)), dtype)
    m = b.ctx.rms_norm(x, w, eps=2.0 ** -126, format="mx8")
    _, Y = rc.norm_exact(b.values(x), b.values(w), 2.0 ** -126)
    got = rc.unpacked(b.raw(m.codes), "mx8")
    fits = np.zeros(got.shape, bool)
    # 64 bits up to the one rounding: nearest for a number within 1e-13 of the exact one
    for f in (1 - 1e-13, 1.0, 1 + 1e-13):
        code, scale, _ = rc.quantize(Y * f, "mx8")
        fits |= np.where(got % 128 == 0, 0, got) == np.where(code % 128 == 0, 0, code)
    assert fits.all(), (int((~fits).sum()), np.argwhere(~fits)[:5].tolist())
    assert np.array_equal(b.raw(m.scales), scale)


# powers of two that the weights lie around: results from the least normal numbers down to where all codes are 0
POWERS = [-126, -131, -136, -137, -140]
