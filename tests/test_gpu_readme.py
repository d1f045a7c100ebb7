"""The README's example: it runs, and what it does around the cache belongs together."""
import os
import re

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_example(gpu_lib):
    with open(os.path.join(ROOT, "README.md")) as f:
        code = re.search(r"```python\n(.*?)```", f.read(), re.S).group(1)
    names = {}
    exec(compile(code, "README.md", "exec"), names)
    torch.cuda.synchronize()
    # tokens behind an eviction go into the same cache as those in front of it, at the positions that they would have without one
    k, v = gpu_lib.kv_cache(16, 128, 8, 128)
    table = torch.arange(16, device="cuda", dtype=torch.int32).view(2, 8)
    want = gpu_lib.rope_kv_append(names["qkv"][:2], names["freq"], k, v, table, names["lens"] + 1, heads=32)
    assert torch.equal(names["q2"], want)
    for name in ("y", "y1", "y2", "y3"):
        assert torch.isfinite(names[name]).all(), name
    assert names["lens2"].tolist() == [128, 78] and names["kept"].shape == (2, 8, 128)
    # what attention adds up of a row's weights is one for each of its heads
    n = names["lens"]
    assert torch.allclose(names["acc"][0, :, : int(n[0])].sum(-1), torch.full((8,), 4.0, device="cuda"), rtol=1e-4)
    assert torch.allclose(names["y2"].float(), names["y1"].float(), rtol=2 ** -7, atol=2 ** -8)      # two roundings to bf16
