"""Gradient of an embedding table on whole numbers: every sum is exact in fp32 (below 2^24), in
any order, so a part that is lost or counted twice shows whatever the length of a row."""
import numpy as np
import pytest
import torch

from paper_2101_11552_gb300 import tfg
from test_gpu_embedding import make_ids

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_11552_gb300 import build
    build.build_library()


def check(ids, rows, f, pad, dtype, seed, offset=0):
    n = len(ids)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    grad = torch.empty(n * f + offset, device="cuda", dtype=dtype)[offset:].view(n, f)
    grad.copy_(torch.randint(-8, 9, (n, f), device="cuda", generator=gen))
    dids = torch.as_tensor(ids).cuda()
    got = tfg.tfg_embedding_backward(tfg.tfg_group_ids(dids, rows, padding_id=pad), grad, 0.5)
    here = torch.ones_like(dids, dtype=torch.bool) if pad is None else dids != pad
    want = torch.zeros(rows, f, dtype=torch.float64, device="cuda").index_add_(0, dids[here], grad[here].double()) * 0.5
    assert float(want.abs().max()) < 2.0 ** 23
    wrong = got.double() != want
    assert not bool(wrong.any()), f"{int(wrong.sum())} of {wrong.numel()} values differ"


@pytest.mark.parametrize("n,rows,f,kind,pad", [
    (1, 1, 1, "uniform", None), (33, 100, 3, "skew", 0), (257, 5, 16, "one", -1), (1000, 119, 128, "skew", None),
    (2049, 3000, 41, "skew", -7), (4097, 2, 100, "one", None), (5000, 20000, 132, "uniform", -1),
    (20000, 119, 64, "skew", None), (20011, 119, 123, "one", 3), (131073, 119, 8, "skew", None),
    (140000, 1000, 12, "one", None), (30000, 700, 300, "skew", None), (9000, 5, 520, "skew", -1),
    (1_000_003, 50, 4, "one", None), (1_000_003, 50, 128, "skew", 7), (300_000, 300_001, 36, "skew", -1),
    (50_000, 3, 1024, "uniform", None), (2000, 40_000, 2000, "skew", None)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient(n, rows, f, kind, pad, dtype):
    ids = make_ids(n, rows, kind, pad, np.random.default_rng(n + f))
    check(ids, rows, f, pad, dtype, n)
    if n * f < 20_000_000:
        check(ids, rows, f, pad, dtype, n + 1, offset=1)                 # off the vector boundary


@pytest.mark.parametrize("f", [4, 16, 60, 128, 130])
def test_rows_that_begin_and_end_everywhere(f):
    """Runs of equal ids of every length around a worker's and a CTA's share."""
    rng = np.random.default_rng(f)
    lengths = np.concatenate([np.arange(1, 40), rng.integers(1, 300, 200), [5000, 1, 4096, 1, 20_000, 2, 70_000]])
    rng.shuffle(lengths)
    ids = np.repeat(np.arange(len(lengths)), lengths)
    check(ids, len(lengths), f, None, torch.float32, f)
    check(rng.permutation(ids), len(lengths) + 5, f, None, torch.bfloat16, f)
