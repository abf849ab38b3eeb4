"""Edges of the 8-bit backbone calls without a GPU."""
import pytest
import torch  # noqa: F401  (before the library: a process has one HIP runtime, torch's)

import paper_2310_18547_amd as sg

FAKE = 0x10000   # a non-null, aligned address that is never dereferenced on these paths
OK, NULL, SHAPE, UNSUPPORTED, ALIGN = 0, 1, 2, 3, 4


@pytest.mark.parametrize("n", [1, 5, 128, 129, 1 << 14, 1 << 20, 1 << 27, 1 << 28, (1 << 28) + 300, (1 << 29) + 8, 1 << 30])
def test_plan_dense_takes_every_batch_within_the_stated_limits(n):
    """Many narrow projections, a wide one beside narrow ones, the widest: the limit is the number of values, not what a launch takes."""
    for h_outs in ([8], [8] * 2, [8] * 8, [16, 8, 8], [72, 8, 264], [1 << 27, 8], [1 << 27] * 8, [1 << 20] * 3):
        for h_in in (8, 4096):
            for nbytes in (0, 16 << 20):
                rc, p = sg.sgmv_plan_dense_q8(sg.F16, n, h_in, h_outs, FAKE if nbytes else None, nbytes, check=False)
                what = (n, h_in, h_outs, nbytes)
                if n * sum(h_outs) > 1 << 38:
                    assert rc == UNSUPPORTED, what
                    continue
                assert rc == OK and p.launches >= 1 and p.workgroups >= 1, what
                # a launch takes fewer than 2^32 threads, a workgroup of these kernels has 192 at least
                assert p.workgroups * 192 <= p.launches * (1 << 32), what


def test_plan_dense_in_several_launches():
    p = sg.sgmv_plan_dense_q8(sg.F16, 1 << 30, 8, [8, 8])
    assert p.launches > 1 and p.slices == 1
    assert sg.sgmv_plan_dense_q8(sg.F16, 1 << 22, 8, [8] * 8).launches == 1
