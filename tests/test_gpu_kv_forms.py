"""Instances of the cache kernels that only larger problems choose."""
import numpy as np
import pytest
import torch

import paper_2311_05161_b200 as w4a8
from kv_util import Batch, encode_block, vectors
from test_gpu_kv_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(8, 8), (16, 2), (24, 2), (32, 2)])
@pytest.mark.parametrize("window", [0, 45])
def test_batches_that_fill_the_gpu(D, Hq, H, window):
    """Four warps per CTA with one tile of eight rows (up to eight query heads per key head) and with two."""
    rng = np.random.default_rng(D + Hq)
    lens = [int(v) for v in rng.integers(0, 200, 100)] + [1500, 0, 1]
    run(lens, None, 16, Hq, H, D, window=window)


@pytest.mark.parametrize("D", [64, 128])
def test_speculative_rows_of_many_sequences(D):
    """Four rows of four heads: two tiles of eight rows, four warps, rows of a sequence across tiles."""
    rng = np.random.default_rng(D)
    lens = [int(v) for v in rng.integers(1, 400, 60)]
    run(lens, [int(v) for v in rng.integers(0, 6, 60)], 32, 16, 4, D, pad=3)


@pytest.mark.parametrize("n,H,D", [(700, 8, 128), (3000, 8, 128), (900, 5, 64), (130, 32, 64), (9000, 3, 64)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_append_of_some_vectors_per_cta(n, H, D, dtype):
    """Every byte of a prompt, where a CTA holds one, some or all of a row's vectors."""
    bt = Batch([n], [n], 64)
    K, V = vectors((n, H, D), 1, dtype, 1.5), vectors((n, H, D), 2, dtype, 0.7)
    cache = w4a8.new_kv_cache(bt.num_pages, 64, H, D).fill_(0x5A)
    ws = w4a8.new_kv_workspace(1, 1, H, H, D)
    w4a8.kv_append(K.cuda(), V.cuda(), cache, bt.table, bt.kv_lens, ws, cu_rows=bt.cu)
    w4a8.check_status(ws)
    got = cache.cpu().numpy().reshape(bt.num_pages, H, 4, 16 * (D + 8))
    sample = np.unique(np.concatenate([np.arange(0, n // 16, max(1, n // 320)), [0, n // 16 - 1]]))
    for blk in sample:
        page, part = bt.table_host[0, blk * 16 // 64], blk % 4
        for h in range(H):
            rows = slice(16 * blk, 16 * blk + 16)
            want = encode_block(K[rows, h].float().numpy(), V[rows, h].float().numpy())
            assert np.array_equal(got[page, h, part], want), (blk, h)
    k, v = w4a8.kv_read(cache, bt.table, bt.kv_lens, n, H, D, ws, cu_rows=bt.cu, dtype=dtype)
    w4a8.check_status(ws)
    from kv_util import quantize_vectors
    for got, x in ((k, K), (v, V)):
        lev, step, _ = quantize_vectors(x.float().numpy())
        assert torch.equal(got.cpu(), torch.from_numpy(lev.astype(np.float32) * step).to(dtype))
