"""The products with contractions long enough for the loops that load ahead, against float64 (tests/moe_ref.py) with the bounds of
tests/test_gpu_moe.py: for each size of tile, even and odd numbers of stages, contractions that end inside a stage, and those that
begin at different stages (multiples of 64, transposed); and inputs whose byte offsets end on either side of 2^31."""
import pytest
import torch

import moe_ref as ref
import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def near(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = (got - want).abs() > bound
    assert not bad.any() and not got.isnan().any(), (what, int(bad.sum()), float((got - want).abs().max()))


def bound(K, size, want, dtype):
    return 2 * (K + 8) * ref.U32 * size + want.abs() * (ref.UBF if dtype == BF else ref.U32) + 1e-38


# T, E, k, columns of the result: tiles of 256 x 256, 128 x 256, 64 x 256, 64 x 128
TILES = [(4096, 2, 2, 4104), (2100, 16, 2, 4104), (1000, 64, 1, 2056), (100, 4, 2, 136)]
# stages of 32: 20, 22, 10 and a quarter, 21; of 64 (transposed): 10, 11, 5 and an eighth, 10 and a half
LENGTHS = [640, 704, 328, 672]


def check(T, E, k, K, cols, transpose):
    n, m = (cols, K) if transpose else (K, cols)
    g = torch.Generator().manual_seed(T + K)
    experts = ref.draw_experts(T, E, k, g, none=0.03)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, _ = ref.rows(experts, E)
    w = torch.randn(E, n, m, generator=g).to(BF)
    scale = torch.randn(T, k, generator=g)
    for gather, dtype, s in ((True, BF, None), (False, F32, scale)):
        x = torch.randn(T if gather else T * k, K, generator=g).to(BF)
        kw = dict(gather=gather, transpose=transpose, scale=s)
        want, size = ref.matmul(x, w, off, row, k, **kw), ref.matmul(x, w, off, row, k, absolute=True, **kw)
        args = (x.to(DEV), w.to(DEV), plan)
        kw = dict(gather=gather, transpose=transpose, scale=None if s is None else s.to(DEV), dtype=dtype)
        got = P.expert_matmul(*args, **kw)
        near(got, want, bound(K, size, want, dtype), (gather, dtype))
        assert torch.equal(got, P.expert_matmul(*args, **kw))


@pytest.mark.parametrize("transpose", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("K", LENGTHS)
@pytest.mark.parametrize("tile", TILES, ids=lambda c: "x".join(map(str, c)))
def test_long_contractions(tile, K, transpose):
    T, E, k, cols = tile
    check(T, E, k, K, cols, transpose)


@pytest.mark.parametrize("transpose", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("case", [(1000, 16, 1, 4096, 520), (900, 16, 1, 4100, 520), (2100, 16, 2, 641, 4101), (100, 4, 2, 675, 131),
                                  (900, 16, 1, 4101, 519)], ids=lambda c: "x".join(map(str, c)))
def test_shared_contractions_and_any_length(case, transpose):
    check(*case, transpose)


# T, E, k, n, m: tiles of 256 x 256 with several lists of places, 128 x 256, 64 x 128; the last two of any length
@pytest.mark.parametrize("case", [(2600, 2, 1, 4200, 4360), (1300, 8, 2, 1024, 2056), (4000, 2, 1, 136, 264), (1300, 8, 2, 1023, 2055),
                                  (4000, 2, 1, 131, 259)], ids=lambda c: "x".join(map(str, c)))
def test_weights_gradient_of_many_rows(case):
    T, E, k, n, m = case
    g = torch.Generator().manual_seed(T + n)
    experts = ref.draw_experts(T, E, k, g, none=0.03)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, _ = ref.rows(experts, E)
    K = int((off[1:] - off[:-1]).max())
    dy = torch.randn(T * k, m, generator=g).to(BF)
    for gather in (False, True):
        x = torch.randn(T if gather else T * k, n, generator=g).to(BF)
        want, size = (ref.matmul_grad(x, dy, off, row, k, gather, absolute=a) for a in (False, True))
        got = P.expert_matmul_grad(x.to(DEV), dy.to(DEV), plan, gather=gather)
        near(got, want, bound(K, size, want, BF), gather)
        assert torch.equal(got, P.expert_matmul_grad(x.to(DEV), dy.to(DEV), plan, gather=gather))


@pytest.mark.parametrize("T", [16382, 16383, 16384, 33000], ids=["below", "first above", "at", "above 2^32"])
def test_offsets_on_either_side_of_31_bits(T):
    """Rows of 64 values, 2^17 bytes apart: up to 16382 of them lie below 2^31 with one to spare."""
    ld, E, n, m = 1 << 16, 4, 64, 72
    g = torch.Generator().manual_seed(T)
    room = torch.zeros(T, ld, dtype=BF, device=DEV)
    x = room[:, 8:8 + n]
    values = torch.randn(T, n, generator=g).to(BF)
    x.copy_(values)
    experts = torch.randint(0, E, (T, 1), generator=g, dtype=torch.int32)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, _ = ref.rows(experts, E)
    w, dy = torch.randn(E, n, m, generator=g).to(BF), torch.randn(T, m, generator=g).to(BF)
    K = int((off[1:] - off[:-1]).max())
    for gather in (True, False):
        kw = dict(gather=gather)
        want, size = ref.matmul(values, w, off, row, 1, **kw), ref.matmul(values, w, off, row, 1, absolute=True, **kw)
        near(P.expert_matmul(x, w.to(DEV), plan, gather=gather), want, bound(n, size, want, BF), gather)
        want, size = (ref.matmul_grad(values, dy, off, row, 1, gather, absolute=a) for a in (False, True))
        near(P.expert_matmul_grad(x, dy.to(DEV), plan, gather=gather), want, bound(K, size, want, BF), gather)
