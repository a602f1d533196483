"""CPU: which form a 4-bit product takes, and what the query refuses."""
import pytest

import paper_2501_07161_b200 as q


@pytest.mark.parametrize("m,n,groups,form,tiles", [(1, 4096, 1, 16, 32), (17, 128, 1, 32, 1), (64, 4096, 1, 64, 32), (333, 1000, 1, 32, 88),
                                                   (640, 1700, 1, 64, 140), (1200, 1100, 1, 128, 90), (5000, 2100, 1, 256, 180),
                                                   (64, 4096, 32, 16, 1152), (4495, 2100, 8, 256, 234), (0, 5, 1, 16, 0), (5, 0, 1, 16, 0)])
def test_form_of_a_product(m, n, groups, form, tiles):
    assert q.mx_form(m, n, groups, 148) == (form, tiles)


def test_every_row_is_covered():
    """The form's tiles cover all rows however they fall into groups, and only the widest form has more than one per SM of a
    dense product of more than 64 rows."""
    for m in (1, 16, 17, 33, 65, 128, 500, 1000, 4097, 1 << 20):
        for n in (1, 128, 129, 4096):
            for groups in (1, 3, 512):
                form, tiles = q.mx_form(m, n, groups, 148)
                assert tiles >= -(-m // form) * -(-n // (256 if form == 256 else 128))
                assert form == 256 or tiles <= 148 or -(-m // groups) <= 64


@pytest.mark.parametrize("args,status", [((1, 1, 0, 148), -1), ((1, 1, 1, 0), -1), (((1 << 30) + 1, 1, 1, 148), -4), ((1, (1 << 30) + 1, 1, 148), -4),
                                         ((1, 1, 513, 148), -4)])
def test_refusals(args, status):
    with pytest.raises(q.binding.Qv2Error) as e:
        q.mx_form(*args)
    assert e.value.status == status
