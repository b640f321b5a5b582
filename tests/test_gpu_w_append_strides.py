"""New rows into caches that lie among other things: pages of one layer of several, K and V of a slot side by side, rows with room behind their heads."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests.test_gpu_r_pages import F8, Rows      # noqa: E402

# few rows, and enough of long prompts for the kernel of those (2**18 or 2**17 heads of rows)
SEQS = {"few": dict(seqs=[(5, 3), (0, 40), (31, 1), (16, 17)], hq=6, hkv=3), "many": dict(seqs=[(5, 4000), (33, 4300)], hq=16, hkv=8)}


@pytest.mark.parametrize("d, dtype", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("seqs", SEQS)
def test_pages_of_one_layer_among_others(seqs, d, dtype):
    r = Rows(cache="8bit", d=d, dtype=dtype, **SEQS[seqs])
    # layers of a page side by side, and a free KV head's room behind them
    total, hkv = r.pages.shape[:2]
    store = torch.full((total, 3 * hkv + 1, 2, 16, d), 0x55, dtype=torch.uint8, device="cuda").view(F8)
    mine = store[:, hkv:2 * hkv]
    mine.copy_(r.pages)
    r.pages = r.kw["pages"] = mine
    r.run()
    r.check()
    assert (store.view(torch.uint8)[:, :hkv] == 0x55).all() and (store.view(torch.uint8)[:, 2 * hkv:] == 0x55).all()


@pytest.mark.parametrize("cache", ["pages", "slots"])
@pytest.mark.parametrize("d, dtype", [(128, "f16"), (64, "bf16")])
@pytest.mark.parametrize("seqs", SEQS)
def test_keys_and_values_of_a_slot_side_by_side(seqs, cache, d, dtype):
    r = Rows(cache=cache, d=d, dtype=dtype, **SEQS[seqs])
    slots, hkv = r.pool[0].shape[:2]
    store = torch.full((slots, 2 * hkv * d + 24), 5.0, dtype=r.pool[0].dtype, device="cuda")
    at = store[:, 8:8 + 2 * hkv * d].view(slots, 2, hkv, d)
    at[:, 0], at[:, 1] = r.pool[0], r.pool[1]
    r.pool = [at[:, 0], at[:, 1]]
    r.kw["k_pool"], r.kw["v_pool"] = r.pool
    r.run()
    r.check()
    assert (store[:, :8] == 5).all() and (store[:, 8 + 2 * hkv * d:] == 5).all()


@pytest.mark.parametrize("cache", ["8bit", "pages"])
@pytest.mark.parametrize("seqs", SEQS)
def test_rows_with_strides_of_their_own(seqs, cache):
    """Queries, keys, values and the queries' results each with another stride."""
    r = Rows(cache=cache, packed=False, **SEQS[seqs])

    def wide(x, more):
        rows, heads, d = x.shape
        y = torch.full((rows, heads * d + more), 9.0, dtype=x.dtype, device="cuda")
        y[:, :heads * d] = x.reshape(rows, -1)
        return y.as_strided((rows, heads, d), (heads * d + more, d, 1)), y[:, heads * d:]

    rest = []
    for name, more in (("q", 8), ("k", 16), ("v", 136), ("q_out", 40)):
        x, behind = wide(getattr(r, name), more)
        setattr(r, name, x)
        rest.append(behind)
    r.run()
    r.check()
    assert all((x == 9).all() for x in rest)
