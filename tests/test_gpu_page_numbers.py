"""Page numbers out of range that are handed on: a call that takes one from the ring, or gives one back to it, says so."""
import pytest

from tests.test_gpu_page_assign import World, dev, xkv  # noqa: F401  (the fixture)
from tests import _cache8_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [-1, 20, 1 << 30, -(1 << 31)])
@pytest.mark.parametrize("batch", [2, 1500])
def test_out_of_range(xkv, bad, batch):  # noqa: F811
    for where in ("table", "ring", "nowhere"):
        w = World(xkv, 16, batch * 8 + 12, 6, batch)
        bad_id = w.n_pages if bad == 20 else bad
        held = w.call([0] * batch, [40, 16] + [0] * (batch - 2))
        if where == "table":
            w.table[0][1] = bad_id
            w.d[0].copy_(dev(w.table))
        if where == "ring":
            w.ring[(w.state[0] + 2) % w.n_pages] = bad_id
            w.d[1].copy_(dev(w.ring))
        # the first gives two pages back, the second takes four, nobody has tokens placed (no new slots are asked for)
        want = [10, 80] + [0] * (batch - 2)
        h, t = dev(held), dev(want)
        length = dev([0] * batch)
        w.flags.zero_()
        w.x.xkv_page_assign(w.cfg, h, t, *w.d, None, length, flags=w.flags)
        table, ring, state, _, length_r, _, _, _ = R.assign_ref(16, w.n_pages, 6, held, want, w.table, w.ring, w.state, 0)
        assert w.d[0].tolist() == table and w.d[1].tolist() == ring and w.d[2].tolist() == state and length.tolist() == length_r
        assert int(w.flags) == (0 if where == "nowhere" else xkv.XKV_FLAG_INDEX_RANGE), where
