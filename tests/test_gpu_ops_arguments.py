"""Arguments that the Python functions of the operators refuse before anything is launched."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def test_status_is_one_int32(dare):
    """The kernels write four bytes there."""
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    x = torch.randn((4, 2, 64), device="cuda").bfloat16()
    w = torch.randn((32, 64), device="cuda").bfloat16()
    table = dare.rope_table(16, 64, 1e4)
    calls = (lambda s: dare.rope(x, table, status=s), lambda s: dare.linear(x[:, 0], w, status=s),
             lambda s: dare.attention(x, x, x, ints([0, 4]), ints([0, 4]), status=s))
    for call in calls:
        for bad in (torch.zeros(1, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"),
                    torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32)):
            with pytest.raises(ValueError):
                call(bad)
        good = ints([0])
        call(good)
        assert good.item() == dare.OK
