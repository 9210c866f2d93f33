"""Units that are fewer than CTAs and yet cut as one list: more than 32 sequences, more than three tiles of query rows, parts that do not fit."""
import pytest
import torch

import cache_plain as cp
from test_gpu_cache_attend import check

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,Hq,Hkv,D", [(1, 2, 1, 64), (1, 8, 2, 128), (3, 4, 1, 64), (9, 8, 1, 128), (20, 8, 1, 64), (1, 2, 1, 192)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 5)])
def test_more_than_32_sequences(dtype, n, Hq, Hkv, D, window, sinks):
    for lens in ([n + i % 3 for i in range(33)],                                  # a tile each
                 [n] * 70 + [2500],                                               # one long one behind short ones
                 [1800] + [n + 7] * 40 + [n + 129, 300, n],
                 [n + 137 * (i * 11 % 13) for i in range(36)]):
        c = cp.make(len(lens), n, Hq, Hkv, D, 16, lens, dtype=dtype, seed=len(lens))
        check(c, window=window, sinks=sinks)
        # only some of them bring tokens, so that the list is shorter than there are CTAs
        new = torch.tensor([n if i % 9 == 0 else 0 for i in range(len(lens))], dtype=torch.int32, device="cuda")
        check(c, n_new=new, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,n,Hq,Hkv,lens", [(1, 100, 8, 1, [100]), (1, 300, 1, 1, [700]), (2, 130, 4, 1, [131, 900]), (1, 41, 8, 1, [2000]), (31, 2, 8, 4, [2 + 90 * i for i in range(31)])])
def test_many_tiles_of_rows_and_parts_that_do_not_fit(dtype, B, n, Hq, Hkv, lens):
    c = cp.make(B, n, Hq, Hkv, 64, 16, lens, dtype=dtype, seed=n)
    check(c)
    check(c, window=77, sinks=3)
