"""Windows and first tokens as Python has them, of any size, reach the library as the nearest that an int32 holds."""
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_attend_abi import Ctx, library, on_gpu  # noqa: F401

MOST, LEAST = 2 ** 31 - 1, -2 ** 31


@pytest.mark.parametrize("given,handed", [(7, 7), (0, 0), (-3, -3), (MOST, MOST), (MOST + 1, MOST), (1 << 40, MOST), (LEAST, LEAST), (LEAST - 1, LEAST),
                                          (-(1 << 32), LEAST), (-(1 << 40) + 5, LEAST)])
def test_windows_and_first_tokens(library, given, handed):  # noqa: F811
    cache = B.Cache(on_gpu(4, 2, 16, 64), on_gpu(4, 2, 16, 64))
    seqs = B.Sequences(3, on_gpu(3, 5, dtype=torch.int32), on_gpu(3, dtype=torch.int32))
    q, out = on_gpu(3, 256), on_gpu(3, 256)
    B.as_attend(Ctx, cache, seqs, q, out, window=given, sinks=given)
    B.as_attend_prompts(Ctx, cache, seqs, q, on_gpu(4, dtype=torch.int64), out, window=given, sinks=given)
    for _, args in library.calls:
        assert args[-4:-2] == (handed, handed)
