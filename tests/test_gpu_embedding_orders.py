"""The order of the tokens behind the embeddings' gradient, for every number of sorting passes, and sums of frequent tokens that go
through pieces of every length.

Against 64 bits: a sum of m floats in any order is off by (m + 1) 2^-24 times the sum of their magnitudes, and the scale's
product by one rounding more."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_encoder import BF16, F32, clean_status, close, gen, gs, normal, padded  # noqa: E402, F401


@pytest.mark.parametrize("n", [4000, 9001])                         # by one thread block in one launch, by several
@pytest.mark.parametrize("vocabulary", [500, 512, 2 ** 18 - 1, 2 ** 18, 2 ** 27 - 1, 2 ** 27 + 5])        # (keys run to the vocabulary's size: 9, 10, 18, 19, 27 and 28 bits)
def test_every_number_of_passes(gs, n, vocabulary):  # noqa: F811
    g = gen(n + vocabulary % 1000)
    ids = torch.randint(-1, vocabulary, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[n // 3:n // 2] = ids[:n // 2 - n // 3]                       # (tokens that occur again)
    ids[-3:] = torch.tensor([vocabulary - 1, 0, -1], dtype=torch.int32)
    d_out, d_table = normal(n, 3, F32, g), padded(vocabulary, 3, F32)
    gs.embedding_backward(d_out, ids, d_table, scale=2.0)
    there = ids >= 0
    token, at = torch.unique(ids[there].long(), return_inverse=True)
    zero = torch.zeros(len(token), 3, dtype=torch.float64, device="cuda")
    rows = d_out.double()[there] * 2.0
    want, size = zero.index_add(0, at, rows), zero.index_add(0, at, rows.abs())
    terms = torch.bincount(at, minlength=len(token))[:, None]
    close(d_table[token], want, (terms + 2) * 2.0 ** -24 * size)
    d_table[token] = 0.0
    assert not d_table.any()                                         # every other row is zero
    assert gs.device_status() == 0


@pytest.mark.parametrize("n", [65536, 65537, 262144, 262145])       # pieces of 16, 64, 64 and 128 places
@pytest.mark.parametrize("repeat", [1, 2, 40, 90, 1000, 20000])
def test_runs_of_every_length(gs, n, repeat):  # noqa: F811
    """Every token `repeat` times in a row of the sorted list, at places that no piece's length divides; in whole numbers, exact."""
    g = gen(n + repeat)
    vocabulary = (n + 7) // repeat + 1
    order = torch.randperm(n, generator=g, device="cuda")
    ids = ((torch.arange(n, device="cuda") + 7) // repeat).to(torch.int32)[order]
    d_out = padded(n, 24, BF16)
    d_out.copy_(torch.randint(-8, 9, (n, 24), generator=g, device="cuda"))
    d_table = padded(vocabulary, 24, F32)
    gs.embedding_backward(d_out, ids, d_table)
    want = torch.zeros(vocabulary, 24, dtype=torch.float64, device="cuda").index_add(0, ids.long(), d_out.double())
    assert torch.equal(d_table.double(), want)
    assert gs.device_status() == 0
