"""4-bit weights with group scales: packing, unpacking and products with a few rows, against their definitions in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

import w4_helpers as R
from paper_2605_05888_b200 import binding as B

gpu = pytest.mark.gpu


# ---- on the CPU: refusals, and the form itself -----------------------------------------------------------------------------

@pytest.fixture(scope="module")
def lib():
    import __graft_entry__ as entry
    entry.build()
    return B.lib()


def test_codes_hold_eight_columns_per_word_even_ones_in_the_low_half():
    q = torch.tensor([[1, -3, 2, -4, 3, -5, 4, -6]])
    word = R.encode(q).numpy().view("<u4")[0, 0]
    assert [(int(word) >> (4 * i) & 15) - 8 for i in range(8)] == [1, 2, 3, 4, -3, -4, -5, -6]
    assert torch.equal(R.decode(R.encode(q)), q.double())


def test_calls_refuse_what_they_cannot_take(lib):
    """Every check answers before anything is launched (the addresses are never read)."""
    a = 1 << 20
    good = B.W4T(a, a)

    def matvec(experts=1, N=8, C=128, group=32, w=good, M=1, x=a, ids=None, y=a):
        return lib.moe_w4_matvec(experts, N, C, group, ctypes.byref(w) if w is not None else None, M, x, ids, y, None)

    def pack(dtype=1, experts=1, N=8, C=128, group=32, w=a, out=good):
        return lib.moe_w4_pack(dtype, experts, N, C, group, w, ctypes.byref(out) if out is not None else None, None)

    def unpack(dtype=1, experts=1, N=8, C=128, group=32, w=a, out=good):
        return lib.moe_w4_unpack(dtype, experts, N, C, group, ctypes.byref(out) if out is not None else None, w, None)

    for call in (matvec, pack, unpack):
        assert call(experts=0) == call(N=0) == call(C=0) == call(C=-128) == -1
        assert call(C=96, group=64) == call(C=130) == call(C=64, group=128) == -1     # the group does not divide C
        assert call(group=16) == call(group=0) == call(group=256) == call(group=48, C=96) == -3
    assert matvec(w=None) == matvec(w=B.W4T(None, a)) == matvec(w=B.W4T(a, None)) == -1
    assert matvec(w=B.W4T(a + 8, a)) == matvec(w=B.W4T(a, a + 2)) == matvec(x=a + 8) == matvec(y=a + 4) == matvec(ids=a + 2) == -2
    assert matvec(M=-1) == matvec(x=None) == matvec(y=None) == -1
    assert matvec(experts=65536, ids=a) == matvec(N=(1 << 25) + 1) == matvec(C=1 << 26) == pack(C=1 << 26) == unpack(C=1 << 26) == -3
    assert matvec(experts=2) == -1                                                       # several matrices, no ids
    assert matvec(M=(1 << 30) + 1) == matvec(N=(1 << 30) + 1) == pack(N=(1 << 30) + 1) == unpack(N=(1 << 30) + 1) == -3
    assert matvec(M=0, x=None, y=None) == 0
    for call in (pack, unpack):
        assert call(dtype=2) == call(dtype=-1) == call(w=None) == call(out=None) == -1
        assert call(w=a + 4) == call(out=B.W4T(a + 4, a)) == -2


def test_product_in_the_place_of_its_rows_is_refused(lib):
    """Other threads' rows are still being read when the first results are written."""
    a = 1 << 20
    for M in (1, 3, 17):
        for experts, ids in ((1, None), (4, a)):
            assert lib.moe_w4_matvec(experts, 128, 128, 32, ctypes.byref(B.W4T(a, a)), M, a, ids, a, None) == -1


def test_matrices_that_do_not_belong_together_are_refused():
    u8, bf = torch.uint8, torch.bfloat16
    w = B.W4(torch.zeros(3, 5, 64, dtype=u8), torch.zeros(3, 4, 5, dtype=bf))
    assert (w.experts, w.N, w.C, w.group) == (3, 5, 128, 32)
    for codes, scales in ((torch.zeros(5, 64, dtype=bf), torch.zeros(4, 5, dtype=bf)), (torch.zeros(5, 64, dtype=u8), torch.zeros(4, 5)),
                          (torch.zeros(5, 64, dtype=u8), torch.zeros(4, 6, dtype=bf)), (torch.zeros(5, 64, dtype=u8), torch.zeros(3, 5, dtype=bf)),
                          (torch.zeros(2, 5, 64, dtype=u8), torch.zeros(3, 4, 5, dtype=bf)), (torch.zeros(64, dtype=u8), torch.zeros(4, dtype=bf)),
                          (torch.zeros(5, 64, dtype=u8), torch.zeros(0, 5, dtype=bf))):
        with pytest.raises(ValueError):
            B.W4(codes, scales)
    x, y = torch.zeros(2, 128, dtype=bf), torch.zeros(2, 5, dtype=bf)
    ids = torch.zeros(2, dtype=torch.int32)
    for args in ((x.float(), ids, y), (x, ids, y.float()), (x[:, :64], ids, y), (x, ids, y[:, :4]), (x, ids[:1], y), (x, ids.long(), y)):
        with pytest.raises(ValueError):
            B.moe_w4_matvec(w, *args)
    dense = torch.zeros(3, 5, 128, dtype=bf)
    for call in (lambda: B.moe_w4_matvec(w, x, ids, y), lambda: B.moe_w4_pack(dense, w), lambda: B.moe_w4_unpack(w, dense)):  # all of it in host memory
        with pytest.raises(ValueError):
            call()
    for args in ((x.to("meta"), ids, y), (x, ids.to("meta"), y), (x, ids, y.to("meta"))):
        with pytest.raises(ValueError):
            B.moe_w4_matvec(w, *args)
    with pytest.raises(ValueError):
        B.moe_w4_pack(torch.zeros(3, 5, 64), w)
    with pytest.raises(ValueError):
        B.moe_w4_unpack(w, torch.zeros(3, 5, 128, dtype=torch.float16))


# ---- packing ---------------------------------------------------------------------------------------------------------------

def pack_reference(w: np.ndarray, group: int):
    """(q, scales [E, C/g, N] as float64) by the definition."""
    E, N, C = w.shape
    v = w.astype(np.float64).reshape(E, N, C // group, group)
    fine = np.isfinite(v).all(-1)
    amax = np.where(fine, np.abs(np.where(np.isfinite(v), v, 0)).max(-1), 0)
    quotient = (amax.astype(np.float32) / np.float32(7)).astype(np.float32)
    s = torch.from_numpy(quotient).to(torch.bfloat16).double().numpy()
    q = np.where(s[..., None] > 0, np.rint(np.where(fine[..., None], v, 0) / np.where(s > 0, s, 1)[..., None]), 0).clip(-8, 7)
    q = np.where(fine[..., None], q, 0)
    s = np.where(fine, s, np.nan)
    return q.reshape(E, N, C), s.transpose(0, 2, 1)


def check_pack(w: torch.Tensor, group: int):
    E, N, C = w.shape
    q, s = pack_reference(w.float().cpu().numpy(), group)
    # room behind both outputs that has to stay as it was
    codes = torch.full((E * N * C // 2 + 64,), 0xa5, dtype=torch.uint8, device="cuda")
    scales = torch.full((E * N * C // group + 64,), 123.0, dtype=torch.bfloat16, device="cuda")
    out = B.W4(codes[:E * N * C // 2].view(E, N, C // 2), scales[:E * N * C // group].view(E, C // group, N))
    B.moe_w4_pack(w, out)
    assert np.array_equal(R.decode(out.codes).cpu().numpy(), q)
    assert np.array_equal(out.scales.double().cpu().numpy(), s, equal_nan=True)
    assert (codes[E * N * C // 2:] == 0xa5).all() and (scales[E * N * C // group:] == 123.0).all()
    for dt in (torch.bfloat16, torch.float32):
        back = torch.full((E * N * C + 64,), 7.0, dtype=dt, device="cuda")
        B.moe_w4_unpack(out, back[:E * N * C].view(E, N, C))
        want = torch.from_numpy(q).cuda() * torch.from_numpy(s).cuda().transpose(1, 2).repeat_interleave(group, dim=2)
        assert torch.equal(back[:E * N * C].view(E, N, C).nan_to_num(nan=-1e30), want.float().to(dt).nan_to_num(nan=-1e30))  # (the product has 12 bits: exact in fp32)
        assert (back[E * N * C:] == 7.0).all()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 3, 2), (5, 7, 3), (2, 129, 9), (3, 1001, 16)])
def test_pack_and_unpack(dtype, group, shape):
    E, N, groups = shape
    g = torch.Generator(device="cuda").manual_seed(N * group)
    w = torch.empty(E, N, groups * group, dtype=dtype, device="cuda").normal_(0.0, 0.02, generator=g)
    check_pack(w, group)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,N,C,group", [(2, 3001, 4096, 128), (210, 745, 128, 32), (70001, 2, 32, 32)])
def test_pack_of_more_rows_than_the_grid(dtype, E, N, C, group):
    g = torch.Generator(device="cuda").manual_seed(N)
    check_pack(torch.empty(E, N, C, dtype=dtype, device="cuda").normal_(0.0, 0.02, generator=g), group)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,C,group", [(1, 1 << 25, 128), (3, (1 << 25) - 32, 32), (2, 65535 * 512 + 64, 64), (2, 65535 * 512, 128)])
def test_pack_of_the_longest_rows(dtype, N, C, group):
    """The most columns that the calls take, and both sides of what 65535 segments of 512 columns hold."""
    g = torch.Generator(device="cuda").manual_seed(7)
    w = torch.empty(1, N, C, dtype=dtype, device="cuda").normal_(0.0, 0.02, generator=g)
    out = B.W4(torch.full((1, N, C // 2), 0xa5, dtype=torch.uint8, device="cuda"), torch.full((1, C // group, N), 123.0, dtype=torch.bfloat16, device="cuda"))
    B.moe_w4_pack(w, out)
    groups = w.view(N, C // group, group)
    scales = (groups.abs().amax(-1).double() / 7).float().to(torch.bfloat16)    # (53 bits are enough: the quotient rounds to fp32 as the exact one)
    assert torch.equal(out.scales[0], scales.T)
    back = torch.empty_like(w)
    B.moe_w4_unpack(out, back)
    for n in range(N):
        s = scales[n].double().unsqueeze(-1)
        want = (torch.round(groups[n].double() / s).clamp(-8, 7) * s).flatten()
        assert torch.equal(back[0, n], want.float().to(dtype))


@gpu
def test_matvec_of_the_longest_rows():
    N, C, group = 3, 1 << 25, 128
    g = torch.Generator(device="cuda").manual_seed(8)
    codes = torch.randint(0, 256, (N, C // 2), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.empty(C // group, N, dtype=torch.bfloat16, device="cuda").uniform_(0.5, 1.5, generator=g)
    x = torch.zeros(2, C, dtype=torch.bfloat16, device="cuda")     # few columns that count, so that the sums' roundings stay small
    at = torch.randint(0, C, (500,), device="cuda", generator=g)
    at[:2] = torch.tensor([0, C - 1], device="cuda")
    x[:, at] = torch.empty(2, 500, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    y = torch.empty(2, N, dtype=torch.bfloat16, device="cuda")
    B.moe_w4_matvec(B.W4(codes, scales), x, None, y)
    # a sum's rounding is in proportion to what it has come to: the additions of zeros add none, so the bound counts the 500
    at = at.unique()
    want, bound = R.matvec(torch.stack([R.weights(codes[n:n + 1], scales[:, n:n + 1])[0, at] for n in range(N)]), x[:, at].double())
    R.assert_within(y, want, bound + R.HALF[torch.bfloat16] * (want.abs() + bound), "y")


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pack_on_the_borders_between_codes(dtype):
    """Weights at (k + 1/2) s and one step of their type on either side of it, for scales of every mantissa."""
    rows = []
    for m in range(128):
        s = np.float32(2.0 ** -5 * (1 + m / 128))                     # a bf16 number, so that 7 s packs to the scale s
        k = np.arange(-7, 7) + 0.5
        mid = torch.from_numpy((k * s).astype(np.float32)).to(dtype)
        bits = mid.view(torch.int16 if dtype == torch.bfloat16 else torch.int32)
        near = torch.cat([(bits + d).view(dtype) for d in (-1, 0, 1)])
        rows.append(torch.cat([torch.tensor([7 * s]).to(dtype), near, torch.zeros(64 - 43, dtype=dtype)]))
    w = torch.stack(rows).unsqueeze(0).cuda()
    check_pack(w, 64)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pack_of_zeros_infinities_and_tiny_numbers(dtype):
    w = torch.zeros(1, 8, 128)
    w[0, 1] = torch.linspace(-3e38, 3e38, 128)          # near the largest numbers
    w[0, 2] = torch.linspace(-1e-40, 1e-40, 128)        # subnormal, scale subnormal
    w[0, 3] = 1e-45                                      # the scale rounds to zero
    w[0, 4, 70] = float("inf")
    w[0, 5, 5] = float("nan")
    w[0, 6, 127] = -float("inf")
    w[0, 7] = -torch.linspace(0, 1, 128)
    check_pack(w.to(dtype).cuda(), 64)


# ---- products --------------------------------------------------------------------------------------------------------------

def check_matvec(E, N, C, group, M, ids, seed=0, stream=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes, scales = R.random_w4(g, 0.05, E, N, C, group=group)
    x = torch.empty(M, C, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = B.W4(codes, scales)
    y = torch.full((M * N + 64,), 55.0, dtype=torch.bfloat16, device="cuda")
    got = y[:M * N].view(M, N)
    e = None if ids is None else torch.tensor(ids, dtype=torch.int32, device="cuda")
    B.moe_w4_matvec(w, x, e, got)
    assert (y[M * N:] == 55.0).all()
    full = [0] * M if ids is None else ids
    for i in sorted(set(full)):
        rows = [m for m in range(M) if full[m] == i]
        if not 0 <= i < E:
            assert (got[rows] == 55.0).all()
            continue
        want, bound = R.matvec(R.weights(codes[i], scales[i]), x[rows].double())
        R.assert_within(got[rows], want, bound + R.HALF[torch.bfloat16] * (want.abs() + bound), f"matrix {i}")


@gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,groups", [(1, 1), (7, 2), (33, 3), (150, 5), (1408, 16), (5003, 7), (4736, 40)])
@pytest.mark.parametrize("M", [1, 3, 8, 9, 16, 17, 35])
def test_matvec_one_matrix(group, N, groups, M):
    check_matvec(1, N, groups * group, group, M, None, seed=M)


@gpu
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("ids", [[0], [4, 4], [3, 0, 3, 1, 3, 1, 2, 3, 0, 4, 3], [-1, 2, 5, 2], [7, -9], list(range(5)) * 7,
                                 [2 ** 31 - 1, 1, -2 ** 31]])
@pytest.mark.parametrize("N,groups", [(5, 1), (300, 3), (2817, 9)])
def test_matvec_matrix_per_row(group, ids, N, groups):
    check_matvec(5, N, groups * group, group, len(ids), ids, seed=len(ids))


@gpu
@pytest.mark.parametrize("ids", [[1] * 19 + [0] * 3 + [1] * 10, [2] * 8 + [1] * 9, [0, 1] * 20, [3] * 40 + [-1] * 30 + [3] * 3])
def test_matvec_more_rows_of_a_matrix_than_share_its_reading(ids):
    check_matvec(5, 333, 512, 64, len(ids), ids)


@gpu
@pytest.mark.parametrize("M", [1, 8, 11, 20, 40])
def test_matvec_one_matrix_with_ids(M):
    """One matrix and an id per row: rows with another id are skipped, whatever the rows' number makes of the batch."""
    check_matvec(1, 150, 384, 64, M, [0 if m % 3 else (-1, 1, 0, 7)[m % 4] for m in range(M)], seed=M)


@gpu
def test_matvec_long_columns_of_few_rows():
    check_matvec(1, 3, 128 * 400, 128, 2, None)


@gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [8, 16])
def test_matvec_root_mean_square_error_of_long_rows(group, M):
    """A column left out of 7168 would be 0.012 of a result; the bound per value alone would not show it."""
    N, C = 3000, 7168
    g = torch.Generator(device="cuda").manual_seed(group + M)
    codes, scales = R.random_w4(g, 0.05, N, C, group=group)
    x = torch.empty(M, C, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    B.moe_w4_matvec(B.W4(codes, scales), x, None, y)
    want = x.double() @ R.weights(codes, scales).T
    # (seventeen addends cut off per matrix instruction of sixteen columns, a rounding per group, each of a partial sum that is no larger than the whole
    # in the root mean square; the final rounding, uniform within half a step, and 2 % for the sample)
    bound = R.HALF[torch.bfloat16] / 3 ** 0.5 * 1.02 + (C * 17 / 16 + C / group) * R.U32
    assert (y.double() - want).norm() / want.norm() <= bound < 0.004


@gpu
def test_matvec_codes_beyond_four_gigabytes():
    E, N, C, group = 140, 8192, 8192, 128
    assert E * N * C // 2 > 2 ** 32
    codes = torch.randint(0, 256, (E, N, C // 2), dtype=torch.uint8, device="cuda")
    scales = torch.rand(E, C // group, N, device="cuda").add_(0.5).to(torch.bfloat16)
    x = torch.randn(3, C, device="cuda", dtype=torch.bfloat16)
    y = torch.empty(3, N, device="cuda", dtype=torch.bfloat16)
    B.moe_w4_matvec(B.W4(codes, scales), x, torch.tensor([139, 0, 138], dtype=torch.int32, device="cuda"), y)
    for m, e in ((0, 139), (1, 0), (2, 138)):
        want, bound = R.matvec(R.weights(codes[e], scales[e]), x[m:m + 1].double())
        R.assert_within(y[m:m + 1], want, bound + R.HALF[torch.bfloat16] * (want.abs() + bound), f"matrix {e}")


@gpu
def test_matvec_infinities_and_nan_stay_in_their_row():
    """An infinity in x gives what the products give: infinity by its sign, NaN where the code is 8; other rows and
    other matrices' infinite scales do not matter."""
    g = torch.Generator(device="cuda").manual_seed(3)
    codes, scales = R.random_w4(g, 0.05, 2, 200, 256, group=64)
    scales[1] = float("inf")
    x = torch.empty(4, 256, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    clean = x.clone()
    x[1, 17] = float("inf")
    x[2, 200] = float("nan")
    w = B.W4(codes, scales)
    y, ref = (torch.empty(4, 200, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.moe_w4_matvec(w, clean, torch.zeros(4, dtype=torch.int32, device="cuda"), ref)
    B.moe_w4_matvec(w, x, torch.tensor([0, 0, 0, 0], dtype=torch.int32, device="cuda"), y)
    assert torch.equal(y[0], ref[0]) and torch.equal(y[3], ref[3]) and y[2].isnan().all()
    q = R.decode(codes[0])[:, 17]
    assert y[1][q == 0].isnan().all() and (y[1][q > 0] == float("inf")).all() and (y[1][q < 0] == -float("inf")).all()
    B.moe_w4_matvec(w, clean, torch.tensor([0, 1, 0, 0], dtype=torch.int32, device="cuda"), y)
    assert torch.equal(y[[0, 2, 3]], ref[[0, 2, 3]]) and not y[1].isfinite().any()


@gpu
def test_matvec_row_does_not_depend_on_the_rows_beside_it():
    """A row's result is the same alone and among others: sums run in one order."""
    g = torch.Generator(device="cuda").manual_seed(4)
    codes, scales = R.random_w4(g, 0.05, 1, 999, 640, group=32)
    w = B.W4(codes, scales)
    x = torch.empty(8, 640, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    y = torch.empty(8, 999, dtype=torch.bfloat16, device="cuda")
    B.moe_w4_matvec(w, x, None, y)
    one = torch.empty(1, 999, dtype=torch.bfloat16, device="cuda")
    for m in range(8):
        B.moe_w4_matvec(w, x[m:m + 1], None, one)
        assert torch.equal(one[0], y[m])


@gpu
def test_matvec_and_packing_on_a_stream_and_in_a_graph():
    g = torch.Generator(device="cuda").manual_seed(5)
    dense = torch.empty(2, 300, 256, dtype=torch.bfloat16, device="cuda").normal_(0, 0.05, generator=g)
    w = B.W4.empty(300, 256, 64, experts=2)
    x = torch.empty(5, 256, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    ids = torch.tensor([1, 0, 1, 1, 0], dtype=torch.int32, device="cuda")
    y, back = torch.zeros(5, 300, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(dense)

    def step():
        B.moe_w4_pack(dense, w)
        B.moe_w4_matvec(w, x, ids, y)
        B.moe_w4_unpack(w, back)

    step()
    torch.cuda.synchronize()
    first = y.clone(), back.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_()
        back.zero_()
        step()
    side.synchronize()
    assert torch.equal(y, first[0]) and torch.equal(back, first[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    dense.mul_(-1)
    x.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(back, -first[1]) and torch.equal(y, (-2 * first[0].float()).to(torch.bfloat16))
