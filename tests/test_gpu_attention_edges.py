"""Packed attention where it can go wrong unseen: values that causality hides, in the blocks of keys that a tile takes in part."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(nq, n, heads, kv_heads, hd, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    return rand(nq, heads, hd), rand(n, kv_heads, hd), rand(n, kv_heads, hd)


# Rows of a tile: 256 (many rows), 128 (few rows over many keys), 32 or 8 (CUDA cores), counted over (query, head of the group).
@pytest.mark.parametrize("dtype,hd,heads,kv_heads,nq,n,tile_rows", [
    (BF16, 128, 8, 2, 300, 300, 256), (BF16, 64, 8, 2, 300, 300, 256), (BF16, 64, 4, 4, 700, 741, 256), (BF16, 64, 64, 8, 700, 741, 256), (BF16, 128, 3, 1, 500, 530, 256),
    (BF16, 128, 8, 2, 64, 4010, 128), (BF16, 64, 8, 2, 64, 4010, 128), (BF16, 128, 14, 2, 50, 3001, 128), (BF16, 64, 1, 1, 290, 6000, 128),
    (F32, 64, 4, 2, 100, 133, 32), (F32, 128, 2, 2, 70, 900, 32), (BF16, 256, 4, 1, 40, 77, 32), (BF16, 32, 2, 2, 70, 600, 32)])
def test_values_hidden_from_a_whole_tile(dare, dtype, hd, heads, kv_heads, nq, n, tile_rows):
    """Keys and values behind the last key that a tile's queries see may be anything, the sequence's own among them."""
    group = heads // kv_heads
    q, k, v = make(nq, n, heads, kv_heads, hd, dtype, nq + n)
    call = lambda: dare.attention(q, k, v, ints([0, nq]), ints([0, n]), causal=True, return_lse=True)
    want, want_lse = (t.clone() for t in call())
    assert bool(want.isfinite().all())
    tiles = (nq * group + tile_rows - 1) // tile_rows
    for t in range(tiles - 2, -1, -1):                         # (from the back: what is broken stays so)
        queries = -(-(t + 1) * tile_rows // group)             # of the tiles up to t, the last perhaps shared with the next tile
        seen = queries + n - nq
        v[seen:], k[seen:] = (INF, NAN) if t % 2 else (NAN, INF)
        got, lse = call()
        whole = (t + 1) * tile_rows // group                   # queries that are in no other tile
        assert torch.equal(got[:whole], want[:whole]) and torch.equal(lse[:whole], want_lse[:whole]), t
        assert not bool(got[queries:].isfinite().all())


@pytest.mark.parametrize("dtype,hd,batch", [(BF16, 128, 1750), (BF16, 64, 3000), (F32, 32, 700)])
def test_slices_back_and_forth_past_all_sums(dare, dtype, hd, batch):
    """Offsets that go to the end and back until the units of work pass 2^31: flagged, and nothing is computed."""
    rows, heads = 100000, 8
    q, k, v = (torch.zeros((rows, heads, hd), dtype=dtype, device="cuda") for _ in range(3))
    status, out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full_like(q, 7.0)
    call = lambda b, o: dare.attention(q, k, v, ints([0, rows] * (b // 2)), ints([0] * (b - 1)), k_len=ints([rows] * (b - 1)), out=o,
                                       status=status, return_lse=True)
    call(batch, out)
    assert status.item() == dare.ERR_DEVICE_CHECK
    assert bool((out == 7.0).all())
