"""tl_kv_append refuses outputs (the queries' and the cache's arrays) that overlap an input or one another.  Host only: the
addresses are never read."""
import pytest

import paper_2607_04031_amd as tl
from tests.test_host_serve import addr, append, cache, rope, status

DATA, EXPS = 10 * 64 * 8 * 128, 10 * 64 * 8             # bytes of the test cache's k (v) and k_exp (v_exp)


@pytest.mark.parametrize("what", ["slots", "positions", "inv_freq"])
@pytest.mark.parametrize("out,end", [(4, 5 * 64 * 128 * 2), (0, DATA), (1, DATA), (2, EXPS), (3, EXPS)])
def test_small_inputs(what, out, end):
    """Q_out (addr(8)) and the cache's arrays (addr(0) to addr(3)) over the first and the last word of an input."""
    out = 8 if out == 4 else out
    words = {"slots": 5, "positions": 5, "inv_freq": 64}[what]
    for at in (addr(out), addr(out) + end - 4, addr(out) - 4 * words + 4):
        if what == "slots":
            assert status(append, cache=cache(), slots=at) == tl.TL_EINVAL
        else:
            assert status(append, cache=cache(), rope=rope(**{what: at})) == tl.TL_EINVAL


def test_positions_of_every_axis():
    r = dict(axes=3, sections=(16, 24, 24), positions=addr(8) - 15 * 4 + 4)
    assert status(append, cache=cache(), rope=rope(**r)) == tl.TL_EINVAL


@pytest.mark.parametrize("kw", [dict(v=addr(0)), dict(v=addr(0) + DATA - 16), dict(k_exp=addr(0) + 64), dict(v_exp=addr(0)), dict(k_exp=addr(1)),
                                dict(v_exp=addr(1) + DATA - 16), dict(v_exp=addr(2) + EXPS - 16), dict(k=addr(2) - 16),
                                dict(elem_bytes=2, v=addr(0) + 2 * DATA - 16)])
def test_arrays_of_the_cache(kw):
    assert status(append, cache=cache(**kw)) == tl.TL_EINVAL
