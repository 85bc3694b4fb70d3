"""Trees of drafted tokens without the positions that only the caller knows (no GPU work)."""
import ctypes

from tests.test_paged_refusals import by, lib, some, null, structs, sz


def test_trees_without_positions():
    spd, l = lib()
    c, b = structs({}, {})
    r = spd.spd_rope(4096, 64, 0)
    l.spd_last_error.restype = ctypes.c_char_p
    for seen, positions, said in ((some, null, b"positions"), (some, some, b"NULL"), (null, null, b"NULL")):
        # the model is NULL, which is looked at behind the arguments
        assert l.spd_verify_forward_paged(null, some, by(c), by(b), by(r), positions, seen, some, some, sz(1 << 40), null) == spd.SPD_ERR_INVALID_ARG
        assert said in l.spd_last_error()
