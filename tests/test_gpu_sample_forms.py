"""he_sample_slots where there are rows enough for every compute unit: each number of rows that a workgroup takes, and each size of
workgroup, on both sides of the lines between them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_sample import check, contexts, he, random_params  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# (a workgroup of 512 threads holds 16 tokens each up to n = 2048 and 32 beyond, so eight rows up to 1024, four up to 4096, two up to 8192 and
# one up to 16384; then 1024 threads; and fewer rows while there are not 256 workgroups)
@pytest.mark.parametrize("n,log2N,n_slots,parts", [(1024, 12, 2048, 1), (1025, 12, 2047, 1), (2048, 12, 2048, 1), (2049, 11, 1024, 1), (4096, 10, 511, 2),
                                                   (4097, 10, 512, 1), (8192, 10, 257, 2), (8193, 10, 256, 1), (16384, 10, 256, 1),
                                                   (16385, 10, 256, 1), (32768, 10, 130, 2), (600, 10, 37, 1), (9000, 10, 100, 2)])
def test_many_rows_of_every_length(contexts, n, log2N, n_slots, parts):  # noqa: F811
    rng = np.random.default_rng(n + n_slots)
    ctx = contexts(log2N)
    logits = np.zeros((n, ctx.N // 2, 2))
    logits[:, :n_slots] = rng.normal(0, 2.5, (n, n_slots, 2))
    rows = n_slots * parts
    check(ctx, logits, rng.random(rows), parts, **random_params(rng, rows, n))
