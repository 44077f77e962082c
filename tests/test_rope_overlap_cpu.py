"""Rotary positions whose outputs share memory with an input or with one another, other than in place,
are refused by the C entry points before any CUDA call (tokens are turned in no order)."""
import ctypes

import pytest

from test_rope_cpu import desc, kdn, status  # noqa: F401

B, T, H, HK, D, ES = 2, 8, 4, 2, 64, 2  # as desc has them
ROW, KROW = H * D * ES, HK * D * ES
APART = [(i + 1) << 20 for i in range(4)]  # q, k, qo, ko


def call(kdn, back, at, **over):  # noqa: F811
    q, k, qo, ko = (ctypes.c_void_p(p) for p in at)
    return status(kdn, back, desc(kdn, **over), [q, k, None, None, qo, ko])


@pytest.mark.parametrize("back", [False, True])
def test_refuses_shared_memory(kdn, back):  # noqa: F811
    inv = kdn.KDN_ERR_INVALID_ARG
    size = (B * T * ROW, B * T * KROW) * 2
    for out in (2, 3):
        for other in range(4):
            if other == out:
                continue
            # the same place (but for an output in the place of its own input), reaching into the end, into the start
            for shift in (0, size[other] - 16, 16 - size[out]):
                if shift == 0 and other == out - 2:
                    continue
                at = list(APART)
                at[out] = at[other] + shift
                assert call(kdn, back, at) == inv, (out, other, shift)


@pytest.mark.parametrize("back", [False, True])
def test_refuses_shared_rows_of_a_projection(kdn, back):  # noqa: F811
    """All four in rows of 16 heads: keys' heads among the queries', queries a head further on, a last row that
    meets a first one."""
    inv, ld = kdn.KDN_ERR_INVALID_ARG, 16 * D
    lds = dict(ldq=ld, ldk=ld, ldqo=ld, ldko=ld)
    head = lambda n, row=0: (1 << 20) + (row * 16 + n) * D * ES
    for at in ((head(0), head(4), head(0), head(2)), (head(0), head(4), head(0), head(3)),
               (head(0), head(6), head(1), head(12)), (head(0), head(4), head(5), head(8)),
               (head(0), head(4), head(8), head(11)), (head(0), head(4), head(1, B * T - 1), head(8)),
               (head(0), head(4), head(14, -1), head(8))):
        assert call(kdn, back, at, **lds) == inv, [(p - (1 << 20)) // (D * ES) for p in at]
    # rows of other lengths through one another
    assert call(kdn, back, (head(0), 1 << 26, head(8), 1 << 27), ldq=ld, ldqo=12 * D) == inv
