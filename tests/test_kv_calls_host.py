"""What the Python calls around the key/value cache refuse before they need a GPU."""
import pytest

M = pytest.importorskip("paper_2511_13061_amd")


@pytest.mark.parametrize("geometry", [(2 ** 64 + 4, 16, 2, 64), (4, 2 ** 32 + 16, 2, 64), (4, 16, 2 ** 32 + 2, 64), (4, 16, 2, 2 ** 32 + 64), (4, 16, 2, -2 ** 32 + 64)])
def test_geometries_that_do_not_fit_the_interface(geometry):
    with pytest.raises(ValueError, match="does not fit"):
        M.KvCache(*geometry)


@pytest.mark.parametrize("args", [dict(length=4, rot=2 ** 32 + 64), dict(length=4, rot=64, first=2 ** 64), dict(length=2 ** 64 + 4, rot=64)])
def test_tables_that_do_not_fit_the_interface(args):
    with pytest.raises(ValueError, match="does not fit"):
        M.rope_table(**args)
