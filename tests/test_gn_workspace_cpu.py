"""Device workspace of the group-norm calls over their range (CPU)."""
import math
import random

import pytest

K = pytest.importorskip("paper_1604_06174_amd.ckpt")

MB = 1 << 20


def nbytes(n, hw, c, groups, backward, **kw):
    return K.op_gn_workspace_bytes(K.gn_desc(n, hw, c, groups, **kw), backward)


@pytest.mark.parametrize("n,c,groups", [(16384, 1024, 1), (16384, 4096, 1), (300000, 768, 1), (100000, 520, 1),
                                        (1 << 20, 1000, 2), (8192, 4088, 8), (60000, 2048, 2), (50000, 515, 1)])
@pytest.mark.parametrize("x", [K.TYPE_BF16, K.TYPE_F32])
def test_rows_of_wide_groups_take_a_few_megabytes(n, c, groups, x):
    """Layer norm and others whose groups no wavefront holds: 1024 records of eight
    bytes a channel at most, half as many for 4096 channels."""
    b = nbytes(n, 1, c, groups, True, xtype=x)
    assert b <= 1024 * 8 * min(c, 2048) + 4096, (n, c, groups, b)
    assert nbytes(n, 1, c, groups, False, xtype=x) == 0


def test_workspace_is_bounded_by_the_tensor_or_a_few_megabytes():
    """Random sizes: 17 MB, or a record of eight bytes a channel for every sample of five
    pixels or more (three where the channels are taken one by one), and 64 more."""
    r = random.Random(3)
    for _ in range(20000):
        c = int(2 ** r.uniform(0, 12.5))
        if r.random() < 0.6:
            c = 8 * ((c + 7) // 8)
        groups = r.choice([g for g in range(1, min(c, 64) + 1) if c % g == 0])
        if c // groups > (1024 if c // groups % 8 else 4096):
            continue
        hw = r.choice([1, 1, 2, 3, 4, 5, 8, int(2 ** r.uniform(0, 14))])
        n = int(2 ** r.uniform(0, 17))
        x = r.choice([K.TYPE_BF16, K.TYPE_F32])
        if n * hw * c >= 1 << 35 or n * groups >= 1 << 25:
            continue
        records = 8 / 5 if c % 8 == 0 and math.lcm(c // groups, 8) <= 4096 else 8 / 3
        for backward in (False, True):
            b = nbytes(n, hw, c, groups, backward, xtype=x)
            assert b <= max(17 * MB, records * n * hw * c + 64 * 8 * c + 4096), (n, hw, c, groups, x, backward, b)
