"""The linear layer up to 8 tokens (activations quantised inside the product) where its k range is split over a cluster, at the
edge of what its ring holds, and for aligned and unaligned rows: bit for bit the product of the quantised matrices, and within
the fp32 sums' bound of test_gpu_mx.py of the 64-bit product."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows_of(x, place):
    """x with rows that begin at 32-byte addresses, in the middle of a longer row, or at odd addresses."""
    if place == "dense":
        return x.clone()
    pad, off = {"strided": (16, 16), "odd": (5, 3)}[place]
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device="cuda")
    view = wide[:, off:off + x.shape[1]]
    return view.copy_(x)


def check(m, n, k, dtype, places):
    from paper_2608_21614_b200 import mx
    g = torch.Generator(device="cuda").manual_seed(m * 131 + n + k)
    x = torch.randn(m, k, generator=g, device="cuda").to(TORCH[dtype])
    x[:, 1] *= 40
    w = mx.quantize(torch.randn(n, k, generator=g, device="cuda") * 0.1)
    q = mx.quantize(x)
    want = mx.matmul(q, w, dtype=torch.float32)
    a, b = mx.dequantize(q).double(), mx.dequantize(w).double()
    limit = (k / 64 + 8) * 2.0 ** -23 * (a.abs() @ b.abs().T)
    assert ((want.double() - a @ b.T).abs() <= limit).all()
    linear = mx.Linear(w, m)
    for place in places:
        v = rows_of(x, place)
        out = torch.full((m, n + 3), 7.0, device="cuda")
        got = linear(v, out=out[:, :n])
        assert torch.equal(got, want), place
        assert (out[:, n:] == 7).all()
        assert torch.equal(linear(v, dtype=torch.bfloat16), want.bfloat16())
    assert linear.device_status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [2048, 2016, 4096, 4128, 4100])           # two and four parts, ends inside a run and a block
@pytest.mark.parametrize("m", [1, 3, 8])
def test_split_over_a_cluster(m, k, dtype):
    check(m, 384, k, dtype, ("dense", "strided", "odd"))


@pytest.mark.parametrize("m,n,k", [(8, 384, 11264), (8, 384, 11265), (1, 130, 11232), (5, 384, 20000),     # four parts: 11 stages each, and more
                                   (8, 9600, 2816), (8, 9600, 2817), (2, 9600, 2788)])                      # one part
def test_where_the_ring_just_holds_a_part(m, n, k):
    check(m, n, k, "bf16", ("dense", "odd"))


@pytest.mark.parametrize("m", [9, 16, 17, 64, 65, 130])
def test_split_with_a_quantisation_of_its_own(m):
    check(m, 384, 4096 + 160, "f32", ("dense", "odd"))


@pytest.mark.parametrize("m,n,k", [(200, 16384, 2048), (512, 8191, 1500), (1000, 4096, 2336), (257, 9000, 1056), (2500, 1300, 1312)])
def test_tiles_of_256_tokens_whose_ring_goes_round(m, n, k):
    check(m, n, k, "bf16", ("dense",))


@pytest.mark.parametrize("m,n,k", [(2304, 2300, 2080), (1025, 4096, 3000), (600, 7000, 1700)])
def test_pairs_whose_ring_goes_round(m, n, k):
    check(m, n, k, "f32", ("dense", "odd"))
