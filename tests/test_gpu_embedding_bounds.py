"""Sums of one sign, where every rounding of a row of additions may point the same way: the embedding's gradient within a bound that counts the
additions as the kernels make them.  A run of k places of one row is added up in chunks of 8 to 256 places, one after another, and its chunks
(at most k / 8 + 2) by four waves, then over the waves; small gradients go by runs of 16, or by shares of k / 16 and 16 waves.  In every case
no sum goes through more than min(k, 256) + k / 16 + 16 additions, each off by 2^-24 of a partial sum of at most sum |dy|."""
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd import embedding as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,channels,run", [(40, 24, 8), (1900, 40, 17), (1900, 40, 300), (20000, 64, 250), (140000, 512, 250), (270000, 512, 255), (140000, 512, 4097), (300000, 24, 100000)])
def test_sums_of_one_sign(n, channels, run, dtype):
    dy = (1 + torch.rand(n, channels, generator=torch.Generator().manual_seed(1))).to(dtype).to(DEV)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(2))
    for idx in (torch.arange(n) // run, (torch.arange(n) // run)[order]):
        rows = int(idx.max()) + 1
        got = E.embedding_backward(dy, idx.to(DEV), rows, 1.25, dtype=torch.float32)
        for part in (slice(0, 8), slice(channels - 8, channels)):
            sums = torch.zeros(rows, 8, dtype=torch.float64).index_add_(0, idx, dy[:, part].cpu().double())
            k = torch.bincount(idx, minlength=rows).double().unsqueeze(1)
            additions = k.clamp(max=256) + k / 16 + 16
            ref.close(got[:, part], 1.25 * sums, 1.25 * sums * ref.U * (1.01 * additions + 1) + ref.LEAST[torch.float32])
