"""The training operators' launches at the ends of their ranges, on the CPU: a launch holds fewer than 2^32 work-items."""
import pytest

from tests._launches import launches, program

pytestmark = pytest.mark.skipif(program() is None, reason="hipcc not available")

# rows, H, F: the most rows with widths whose tensors 288 GB can hold, and the widest layers
TRAIN = [(1 << 20, 32768, 512), (1 << 20, 32768, 64), (1 << 20, 64, 32768), (1 << 20, 16384, 16384), (1 << 20, 8192, 28672), (4096, 1 << 18, 64), (4096, 64, 1 << 18),
         (65536, 1 << 18, 512), (1, 1 << 18, 1 << 18), (300, 1 << 18, 1 << 16)]


def items(command):
    for l in launches(command)[0]:
        yield l.kernel, l.grid[0] * l.block, l.grid[1]


@pytest.mark.parametrize("rows,H,F", TRAIN)
@pytest.mark.parametrize("act", [0, 2])
def test_mlp(rows, H, F, act):
    for grads in ("-", "X", "1", "2", "X12"):
        found = list(items(f"train {rows} {H} {F} {act} {rows} {grads}"))
        assert len(found) == 2
        assert all(x < 1 << 32 and y < 1 << 16 for _, x, y in found), found


@pytest.mark.parametrize("command", ["norm 16777216 1 1 1 16777216 {}", "norm 16777216 4096 0 0 16777216 {}", "norm 16777216 16384 1 0 16777216 {}"])
def test_norm(command):
    for d in "fb":
        assert all(x < 1 << 32 and y < 1 << 16 for _, x, y in items(command.format(d)))


@pytest.mark.parametrize("command", ["ortho 1 65536 65536 0 2", "ortho 4096 1024 1024 0 2", "ortho 4096 64 65536 1 2", "ortho 16 65536 8192 1 2"])
def test_ortho(command):
    assert all(x < 1 << 32 and y < 1 << 16 for _, x, y in items(command))


def test_a_product_that_spans_no_transpose_launches_its_tiles():
    """dW1 asks for the transpose of X in the first launch; without it the launch holds the tiles of dZ alone."""
    with_x, without = launches("train 64 512 2048 2 64 X12", "train 64 512 2048 2 64 X2")
    assert with_x[0].grid[0] == without[0].grid[0] + 512 // 64 * (64 // 64)
