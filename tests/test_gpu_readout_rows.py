"""The readout's cross entropy over the row counts of training batches, against float64: the list
of rows in one launch with their copy (up to 1024 rows), by itself (above), in several rounds
(above 8192), and a vocabulary in several pieces."""
import math

import pytest
import torch

import seq_reference as ref
from paper_2412_06355_gb300 import binding

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def inputs(M, V, D, dtype, seed, ignored=0.2):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H = torch.randn((M, D), generator=g, device="cuda").to(DT[dtype])
    W = (torch.randn((V, D), generator=g, device="cuda") * (2 / math.sqrt(D))).to(DT[dtype])
    y = torch.randint(0, V, (M,), generator=g, device="cuda")
    y[torch.rand(M, generator=g, device="cuda") < ignored] = -100
    return H, W, y, torch.rand(M, generator=g, device="cuda") + 0.5


def run(H, W, y, c, dtype, statistics="lse"):
    M, D = H.shape
    cfg = binding.make_xent_config(M, W.shape[0], D, dtype, statistics=statistics,
                                   labels_dtype="i64" if y.dtype == torch.int64 else "i32")
    loss, lse = binding.xent_forward(cfg, H, W, y)
    got = dict(loss=loss, **binding.xent_backward(cfg, H, W, y, lse, c))
    want = ref.xent(H, W, y, -100, c)
    for k in got:
        ref.check(k, got[k], want[k])
    again = binding.xent_backward(cfg, H, W, y, lse, c)
    for k in again:
        assert torch.equal(torch.nan_to_num(again[k]), torch.nan_to_num(got[k])), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("statistics", ["lse", "max_sum"])
@pytest.mark.parametrize("M,V,D", [(1023, 300, 40), (1024, 777, 64), (1025, 777, 65), (2000, 1001, 100),
                                   (8191, 130, 33), (8192, 300, 64), (8193, 300, 40), (17001, 257, 24)])
def test_row_counts(dtype, statistics, M, V, D):
    run(*inputs(M, V, D, dtype, M), dtype, statistics)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keep", ["none", "first", "last", "one", "second round", "last of a round"])
def test_rows_that_are_left_out(dtype, keep):
    """Ignored rows hold infinities; labels out of range stand among them, in 32 bits here."""
    M, V, D = 9000, 150, 40
    H, W, y, c = inputs(M, V, D, dtype, 5, ignored=0.0)
    live = torch.zeros(M, dtype=torch.bool, device="cuda")
    live[{"none": slice(0, 0), "first": slice(0, 1500), "last": slice(M - 1300, M), "one": slice(4321, 4322),
          "second round": slice(8192, M), "last of a round": slice(8190, 8192)}[keep]] = True
    y[~live] = -100
    H[~live] = float("inf")
    y[17], y[8500] = V, -1
    run(H, W, y.int(), c, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_vocabulary_in_several_pieces(dtype):
    M, V, D = 20000, 9001, 40
    cfg = binding.make_xent_config(M, V, D, dtype)
    _, one = binding.dendsn_xent_workspace_size(cfg)
    assert one < M * V * (6 if dtype == "f32" else 4)      # not all of G at once
    run(*inputs(M, V, D, dtype, 6), dtype)
