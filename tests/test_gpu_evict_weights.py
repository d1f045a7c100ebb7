"""The weights that an eviction leaves: bit for bit what they were, signs among them (-0 may come out as 0, and what is no number as another one that is none)."""
import numpy as np
import pytest

from cache_ref import evict
from test_gpu_attention import Batch, dev
from test_gpu_cache_ops import make_weights

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("lens,keep,recent", [([500, 33, 257, 2, 501], 100, 20), ([9000, 300, 5000], 4500, 0), ([50000, 40961], 20000, 1000), ([70, 64], 64, 64)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["signs", "negative"])
def test_signs(gpu_lib, lens, keep, recent, in_place, kind):
    batch = Batch(lens, 64, 2, 2, 96)
    cap = batch.per * 64
    w = make_weights(batch.rng, (len(lens), 2, cap), "signs" if kind == "signs" else "any")
    w = -w if kind == "negative" else w
    out = torch.cat([batch.k, batch.k]), torch.cat([batch.v, batch.v])
    pages, per_out = batch.k.shape[0], -(-keep // 64)
    table = dev(pages + np.arange(len(lens) * per_out).reshape(len(lens), per_out))
    had = torch.from_numpy(w).cuda()
    _, got, kept = gpu_lib.kv_evict(*out, dev(batch.table), dev(lens), had, keep, recent, table, weights_out=had if in_place else None)
    got, kept = got.cpu().numpy(), kept.cpu().numpy()
    for b, n in enumerate(lens):
        for h in range(2):
            at = evict(w[b, h], n, keep, recent)
            assert kept[b, h, : len(at)].tolist() == at
            want, have = w[b, h, at], got[b, h, : len(at)]
            same = ~np.isnan(want) & (want != 0)
            assert np.array_equal(want[same].view(np.int32), have[same].view(np.int32))
            assert np.isnan(have[np.isnan(want)]).all() and (have[want == 0] == 0).all()
            assert kind == "signs" or (want < 0).any()
