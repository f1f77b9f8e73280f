"""What the package hands on: every entry point of the C ABI and every constant that its arguments take."""
import paper_2406_16260_amd as pkg
from paper_2406_16260_amd import binding as B


def test_every_entry_point_is_a_name_of_the_package():
    for name in B.EXPORTS:
        assert getattr(pkg, name) is getattr(B, name), name


def test_every_constant_is_a_name_of_the_package():
    names = [n for n in vars(B) if n.startswith(("DSATTN_ACT_", "DSATTN_FLAG_"))] + ["DSATTN_F32", "DSATTN_BF16", "DSATTN_E4M3"]
    assert len(names) == 12
    for name in names:
        assert getattr(pkg, name) == getattr(B, name), name
