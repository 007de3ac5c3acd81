"""What the one-launch layer's Python calls refuse before anything reaches the library.  Needs no GPU: the plan is a shell without a
handle, which the library answers with "bad argument", so a call that comes that far has passed the checks."""
import pytest
import torch

from paper_2605_05888_b200 import binding as B

T, H, E, K, F = 3, 64, 4, 2, 128
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    import __graft_entry__ as entry
    entry.build()
    return B.lib()


def shell(dtype, T=T, **more):
    plan = B.Plan.__new__(B.Plan)
    plan.cfg = B.make_config(T, H, E, 1, K, F, dtype, **more)
    plan.workspace, plan.handle = torch.empty(0, dtype=torch.uint8), None
    return plan


def dense(dtype):
    return [torch.zeros(T, H, dtype=dtype), torch.zeros(E, H, dtype=dtype), torch.zeros(E), torch.zeros(E, F, H, dtype=dtype), torch.zeros(E, F, H, dtype=dtype),
            torch.zeros(E, H, F, dtype=dtype), torch.zeros(T, H, dtype=dtype)]


def packed():
    def w4(N, C):
        return B.W4(torch.zeros(E, N, C // 2, dtype=torch.uint8), torch.zeros(E, C // 32, N, dtype=BF16))
    a = dense(BF16)
    a[3:6] = [w4(F, H), w4(F, H), w4(H, F)]
    return a


def passes(call, args):
    with pytest.raises(B.MoeError) as err:
        call(*args, stream=0)
    assert err.value.code == -1


def swap(args, i, t):
    return args[:i] + [t] + args[i + 1:]


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_dense_layer(dtype):
    plan, other = shell(B.DTYPE_BF16 if dtype == BF16 else B.DTYPE_FP32), FP32 if dtype == BF16 else BF16
    args = dense(dtype)
    call = plan.moe_layer_few
    passes(call, args)
    passes(call, swap(args, 2, None))
    passes(call, swap(args, 0, args[0].view(T, 1, H)))       # a batch of sequences of one token each
    passes(call, swap(args, 6, args[6].view(1, T, H)))
    passes(call, swap(args, 3, args[3].view(E * F, H)))
    for i in (0, 6):                                          # too few rows, as of a last batch, and too many
        for rows in (1, T - 1, T + 1):
            with pytest.raises(ValueError):
                call(*swap(args, i, torch.zeros(rows, H, dtype=dtype)), stream=0)
    for i in range(7):
        if i == 2:
            continue
        for bad in (args[i].to(other), args[i].to(torch.float16), args[i][..., :-8], args[i][:-1], args[i].transpose(-1, -2), args[i].flatten(), args[i].to("meta")):
            with pytest.raises(ValueError):
                call(*swap(args, i, bad), stream=0)
        passes(call, swap(args, i, None))                     # a missing one is the library's to refuse
        passes(call, swap(args, i, 1 << 20))                  # a raw pointer is taken as it is
    for bad in (torch.zeros(E - 1), torch.zeros(E + 1), torch.zeros(E, dtype=torch.float64), torch.zeros(E, dtype=BF16), torch.zeros(E, device="meta")):
        with pytest.raises(ValueError):
            call(*swap(args, 2, bad), stream=0)


def test_layer_on_4bit_experts():
    plan, args = shell(B.DTYPE_BF16), packed()
    call = plan.moe_layer_few_w4
    passes(call, args)
    for i in (0, 1, 6):
        for bad in (args[i].float(), args[i][..., :-8], args[i][:-1], args[i].flatten(), args[i].to("meta")):
            with pytest.raises(ValueError):
                call(*swap(args, i, bad), stream=0)
    with pytest.raises(ValueError):
        call(*swap(args, 2, torch.zeros(E, dtype=BF16)), stream=0)
    with pytest.raises(ValueError):
        call(*swap(args, 3, args[5]), stream=0)


def test_tensor_parallel_shards_and_an_empty_batch():
    """A plan with TP shards takes the weights of whole experts; of an empty batch no tensor is needed."""
    passes(shell(B.DTYPE_BF16, tp_shards=4).moe_layer_few, dense(BF16))
    empty = shell(B.DTYPE_BF16, T=0)
    for x in (None, torch.zeros(0, H, dtype=BF16), torch.zeros(0)):
        passes(empty.moe_layer_few, [x, *dense(BF16)[1:6], x])
