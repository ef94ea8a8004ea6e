"""The choice of tokens at the borders of its forms: up to 4096 and up to 8192 positions of a row one launch, of 256 and of 512 threads with 16
tokens each; beyond, chunks of 8192.  The form goes by the row's room, the tokens by its length."""
import pytest

from tests.test_gpu_evict import pick, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [4079, 4080, 4081, 4095, 4096, 4097, 4112, 4113, 8175, 8176, 8177, 8191, 8208, 16383, 16384, 16385, 16400])
@pytest.mark.parametrize("share", [0.0, 0.03, 0.5, 0.999, 1.0])
def test_keep_at_the_borders(n, share):
    L = -(-n // 16) * 16
    lens = [n, n - 1, n // 2, 7]
    pick(weights(4, L, n), lens, [int(share * x) for x in lens], sinks=2, recent=3, stride=L)


@pytest.mark.parametrize("room", [4096, 4112, 8192, 8208, 40000, 2 * 1024 * 1024])
@pytest.mark.parametrize("n", [1, 300, 4096])
def test_keep_in_a_wide_row(n, room):
    """A table as wide as the server's longest sequence may become, lengths far below."""
    pick(weights(2, room, n), [n, n // 2], [n // 3, n], sinks=1, recent=4, stride=n)
