"""What the outputs of an MoE layer may be off by on the average (not collected by
pytest).

A bound on every single value has to allow a sum of n products n half steps of fp32 of
the sum of their magnitudes; the errors of an intermediate in bf16, which partly
cancel, stay below that where n is in the thousands.
Root mean squares can: with independent
roundings, uniform within half a step u = 2^-24, a chain of n additions of independent
terms is off by the variance u^2 / 3 times the sum of i / n, u^2 n / 6 relative to the
sum's own.  Gate and up sum d products each and reach the intermediate with a factor
of about 1 (E[silu'^2] var(g) = E[silu^2] for small and for large g alike), the down
product sums three times F.  The gates are off by 2 K + 16 half steps at most
(operator_reference.experts), taken whole.  Four times the root of it all allows for
sums that are not independent.  An intermediate rounded to bf16 (8 bits: 2^-8 of the
value at most, 2^-9 / sqrt(3) and more on the average) is off by 2^-10."""
from __future__ import annotations

import math

from operator_reference import U


def rms_bound(d, F, K):
    return 4 * U * math.sqrt(d / 3 + F / 2 + (2 * K + 16) ** 2)


def rms_error(got, want):
    """Root mean square of the difference over that of the expected values (fp64)."""
    return float((got.double() - want).square().mean().sqrt() / want.square().mean().sqrt())
