"""The MoE layer for a few tokens in one launch, on bf16, fp32 and 4-bit experts, against its definition in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

import w4_helpers as R
from paper_2605_05888_b200 import binding as B

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


class Layer:
    """Random inputs of a layer and what the calls need.  group 0: plain weights."""

    def __init__(self, T, H, E, K, F, dtype=BF16, group=0, renorm=0, bias=False, seed=1, std=0.05, router_std=0.05, **cfg):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.H, self.E, self.K, self.F, self.dtype, self.group, self.renorm = T, H, E, K, F, dtype, group, renorm

        def normal(std, *shape):
            return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)
        self.x, self.wr = normal(1.0, T, H), normal(router_std, E, H)
        self.bias = torch.empty(E, device="cuda").normal_(0.0, 0.5, generator=g) if bias else None
        shapes = ((E, F, H), (E, F, H), (E, H, F))
        if group:
            self.w = [B.W4(*R.random_w4(g, std, *s, group=group)) for s in shapes]
        else:
            self.w = [normal(std, *s) for s in shapes]
        self.plan = B.Plan(B.make_config(T, H, E, 1, K, F, B.DTYPE_FP32 if dtype == FP32 else B.DTYPE_BF16, renormalize=renorm, **cfg))
        self.room = torch.full((T * H + 64,), 55.0, dtype=dtype, device="cuda")
        self.y = self.room[:T * H].view(T, H)

    def call(self, x=None, y=None, plan=None, stream=None):
        plan, x, y = plan or self.plan, self.x if x is None else x, self.y if y is None else y
        (plan.moe_layer_few_w4 if self.group else plan.moe_layer_few)(x, self.wr, self.bias, *self.w, y, stream=stream)
        return y

    def matrix(self, i):
        w = self.w[i]
        return (lambda e: R.weights(w.codes[e], w.scales[e])) if self.group else (lambda e: w[e].double())

    def check(self):
        self.y.fill_(77.0)
        self.call()
        assert self.plan.moe_last_launch_count() == 1
        assert self.plan.moe_last_status() == (0, 0)
        idx = self.plan.layer_tensor(0).long()
        logits, dl, w, y, bound = R.layer(self.x.double(), self.wr.double(), self.bias, self.matrix(0), self.matrix(1), self.matrix(2), self.K,
                                          self.renorm, idx, self.dtype)
        R.check_picks(idx, logits, dl)
        R.assert_within(self.y, y, bound, "y")
        assert (self.room[self.T * self.H:] == 55.0).all()
        assert np.allclose(self.plan.layer_tensor(1).double().cpu().numpy(), w.cpu().numpy(), rtol=1e-3)
        assert torch.equal(self.plan.layer_tensor(3).long().cpu(), torch.bincount(idx.flatten().cpu(), minlength=self.E))
        return self.y


# T, H, E, K, F: one token and sixteen, one expert, as many picks as experts, one used expert and all, H and F that end inside a
# lane's vectors and a block of columns, more and fewer rows than the GPU has warps
BF16_SHAPES = [(1, 8, 1, 1, 8), (1, 2048, 60, 4, 1408), (2, 136, 3, 3, 72), (3, 264, 5, 2, 1000), (4, 1024, 8, 2, 520), (5, 512, 2, 1, 64), (7, 8, 4, 2, 4104),
               (8, 4104, 16, 2, 8), (8, 256, 256, 8, 128), (9, 640, 7, 7, 328), (13, 1000, 33, 5, 248), (16, 768, 64, 6, 1032), (16, 128, 256, 32, 64),
               (16, 7168, 4, 1, 512), (11, 96, 130, 3, 2056)]
FP32_SHAPES = [(1, 4, 1, 1, 4), (1, 1024, 16, 2, 2048), (3, 1020, 16, 2, 2044), (2, 132, 3, 3, 36), (8, 100, 9, 4, 516), (9, 512, 256, 8, 60), (16, 260, 5, 5, 260),
               (16, 68, 64, 16, 12), (6, 2052, 2, 1, 4)]
W4_SHAPES = [(1, 1, 1, 1, 1), (1, 16, 60, 4, 11), (2, 2, 3, 3, 1), (4, 5, 8, 2, 7), (8, 1, 4, 2, 33), (8, 33, 16, 2, 1), (9, 3, 7, 7, 3), (13, 7, 33, 5, 2),
             (16, 6, 64, 6, 9), (16, 2, 256, 32, 1), (16, 56, 4, 1, 4), (5, 4, 2, 1, 4)]


@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("shape", BF16_SHAPES, ids=str)
def test_layer_bf16(shape, renorm):
    Layer(*shape, renorm=renorm, bias=bool(renorm)).check()


@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("shape", FP32_SHAPES, ids=str)
def test_layer_fp32(shape, renorm):
    Layer(*shape, dtype=FP32, renorm=renorm, bias=bool(renorm)).check()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shape", W4_SHAPES, ids=str)
def test_layer_w4(shape, group):
    T, h, E, K, f = shape
    Layer(T, h * group, E, K, f * group, group=group, renorm=group == 64, bias=group == 32).check()


@pytest.mark.parametrize("T", range(1, 17))
@pytest.mark.parametrize("kind", ["bf16", "fp32", "w4"])
def test_every_token_count(T, kind):
    Layer(T, 384, 12, 3, 320, dtype=FP32 if kind == "fp32" else BF16, group=64 if kind == "w4" else 0, seed=T).check()


# more tokens on an expert than an entry holds, by one, by whole entries, all of them; outputs of a row or two per CTA with many terms
# (several CTAs share them), one expert with as many columns as 40 of them
@pytest.mark.parametrize("shape", [(16, 256, 2, 2, 128), (9, 512, 2, 1, 256), (13, 256, 3, 2, 384), (5, 128, 1, 1, 640), (16, 128, 20, 4, 4096),
                                   (12, 384, 16, 6, 2048), (2, 256, 1, 1, 81920)], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "fp32", "w4"])
def test_many_tokens_of_an_expert_and_few_outputs(shape, kind):
    Layer(*shape, dtype=FP32 if kind == "fp32" else BF16, group=128 if kind == "w4" else 0, renorm=1, seed=3).check()


# a row or ten per CTA, or eighteen and a half, of many terms: all CTAs share all outputs, and a number of rows that is no multiple of a tile's
@pytest.mark.parametrize("T,H,E,K,F,kind", [(16, 1000, 16, 6, 4096, "bf16"), (5, 520, 24, 4, 4096, "bf16"), (9, 1500, 16, 4, 2052, "fp32"), (16, 36, 16, 4, 8192, "fp32"),
                                            (16, 2720, 16, 4, 4096, "w4"), (7, 5024, 16, 4, 4096, "w4"), (3, 160, 16, 8, 8192, "w4")])
def test_outputs_that_all_ctas_share(T, H, E, K, F, kind):
    s = Layer(T, H, E, K, F, dtype=FP32 if kind == "fp32" else BF16, group=32 if kind == "w4" else 0, renorm=1, seed=T)
    y = s.check().clone()
    for _ in range(3):
        assert torch.equal(s.call(), y)


# much 4-bit work (its own form of the code) with rows that end inside a chunk of 256 columns, entries of one token to eight
@pytest.mark.parametrize("T,H,E,K,F,group", [(8, 2624, 16, 4, 4160, 64), (16, 2688, 16, 2, 4224, 128), (1, 4128, 16, 12, 4000, 32), (16, 128, 24, 6, 40064, 64)])
def test_much_4bit_work_and_ragged_rows(T, H, E, K, F, group):
    Layer(T, H, E, K, F, group=group, renorm=T % 2, bias=True, seed=T + group).check()


@pytest.mark.parametrize("dtype,group", [(BF16, 0), (FP32, 0), (BF16, 32), (BF16, 128)])
def test_root_mean_square_error_of_long_sums(dtype, group):
    """The bounds per value grow with the sums' lengths; the error over all values holds sums of thousands of terms to what one left out would show
    (1 / sqrt(H) of gate or up, 1 / sqrt(K F) of down: 0.02 and 0.01 here)."""
    T, H, E, K, F = 16, 2048, 4, 2, 4096
    s = Layer(T, H, E, K, F, dtype=dtype, group=group, renorm=1, seed=21)
    got = s.call().double()
    idx = s.plan.layer_tensor(0).long()
    want = R.layer(s.x.double(), s.wr.double(), None, s.matrix(0), s.matrix(1), s.matrix(2), K, 1, idx, dtype)[3]
    # n roundings of at most 2^-23 of a partial sum, whose root mean square is at most the whole sum's, are n 2^-23 of it together (Minkowski):
    # a matrix instruction of sixteen columns cuts off seventeen addends; silu(g) u takes g's error by silu' <= 1.1 where silu is half of g or more,
    # and u's; the tokens' two numbers double the down product's; 1e-5 for the weights and for what the second numbers leave.
    sums = (3.2 * H + 2 * F) * 17 / 16 * R.U32 + 1e-5
    # the final rounding: uniform within half a step, at most HALF / sqrt(3) of a value; 2 % for the sample
    assert (got - want).norm() / want.norm() <= R.HALF[dtype] / 3 ** 0.5 * 1.02 + sums < 0.005


def test_long_bf16_sums_keep_the_accuracy_of_fp32():
    """65536 terms that cancel: what is left of a gate product is its sum's error, and the layer's weights put it into y.  Matrix instructions cut
    off, towards zero, so a sum that goes through a chain of them loses a part of itself with each: such chains end with a chunk of 64 columns."""
    H, F = 65536, 148 * 128                                    # (whole tiles for every warp: nothing else cuts the sums)
    s = Layer(1, 8, 1, 1, 8, seed=2)
    half = torch.empty(H // 2, dtype=BF16, device="cuda").uniform_(0.5, 1.0).mul_(2.0 ** -10)
    tokens = torch.empty(H // 2, dtype=BF16, device="cuda").uniform_(0.5, 1.0)
    tokens[0] = 1.0
    gate, s.x = torch.cat([half, -half.flip(0)]), torch.cat([tokens, tokens.flip(0)]).view(1, H)
    s.wr = torch.zeros(1, H, dtype=BF16, device="cuda")
    s.w = [gate.expand(1, F, H).contiguous(), torch.zeros(1, F, H, dtype=BF16, device="cuda"), torch.zeros(1, H, F, dtype=BF16, device="cuda")]
    s.w[1][0, :, 0] = 2.0                                      # silu(g) 2 is g where g is small
    s.w[2][0, :F].fill_diagonal_(1.0)
    y = s.call(plan=B.Plan(B.make_config(1, H, 1, 1, 1, F, B.DTYPE_BF16)), y=torch.empty(1, H, dtype=BF16, device="cuda"))
    # M: the largest partial sum, reached linearly.  1024 additions of chunks, each rounded to half a step of a sum of M / 2 on average; in each chunk
    # four instructions that cut off seventeen addends, each by a step of at most the chunk's sum of M / 512: 512 + 272 times 2^-24 M.  2 % for silu
    # and the roundings to bf16.
    M = (half.double() * tokens.double()).sum().item()
    assert y[0, :F].double().abs().max().item() <= 1.02 * (512 + 272) * 2.0 ** -24 * M
    assert (y[0, F:] == 0).all()


def kinds(f):
    return pytest.mark.parametrize("dtype,group", [(BF16, 0), (FP32, 0), (BF16, 32), (BF16, 128)])(f)


@kinds
def test_all_tokens_on_one_expert(dtype, group):
    s = Layer(16, 512, 8, 1, 256, dtype=dtype, group=group)
    s.bias = torch.full((8,), float("-inf"), device="cuda")
    s.bias[5] = 0.0
    s.check()
    assert (s.plan.layer_tensor(0) == 5).all()


def test_equal_experts_lowest_index_first():
    s = Layer(6, 1000, 40, 5, 64)
    s.wr[1:] = s.wr[:1]
    s.check()
    assert (s.plan.layer_tensor(0).cpu() == torch.arange(5, dtype=torch.int32)).all()


def test_router_biases_of_the_lowest_values():
    """Experts masked by -inf or by the lowest fp32 number are picked last, in ascending order, with no weight."""
    for low in (float("-inf"), torch.finfo(FP32).min):
        s = Layer(3, 256, 6, 4, 64, bias=True)
        s.bias[[0, 2, 3, 5]] = low
        s.call()
        idx, w = s.plan.layer_tensor(0).cpu(), s.plan.layer_tensor(1).cpu()
        assert all(sorted(r[:2].tolist()) == [1, 4] and r[2:].tolist() == [0, 2] for r in idx)
        assert (w[:, 2:] == 0).all() and np.allclose(w.sum(1).numpy(), 1.0, atol=1e-6)
        assert s.y.isfinite().all()


@kinds
def test_nan_and_infinity_stay_with_their_token(dtype, group):
    """A token that holds a NaN or an infinity, and an expert with a weight that is not finite, leave the other tokens alone."""
    s = Layer(12, 512, 16, 2, 256, dtype=dtype, group=group, seed=8)
    want = s.call().clone()
    x = s.x.clone()
    x[3, 100] = float("nan")
    x[7, 511] = float("inf")
    y = torch.zeros_like(want)
    s.call(x=x, y=y)
    assert y[3].isnan().all() and not y[7].isfinite().all()
    # The two tokens' picks are others now, so the shares of the warps, and with them the order of a sum, may be: every
    # other token is held to the definition, by the bound on sums in any order.
    rest = [t for t in range(12) if t not in (3, 7)]
    idx = s.plan.layer_tensor(0).long()[rest]
    logits, dl, _, ref, bound = R.layer(x[rest].double(), s.wr.double(), None, s.matrix(0), s.matrix(1), s.matrix(2), 2, 0, idx, dtype)
    R.check_picks(idx, logits, dl)
    R.assert_within(y[rest], ref, bound, "other tokens")
    s.call()
    idx = s.plan.layer_tensor(0).cpu()
    e = int(idx[0, 0])
    for i, name in enumerate(("gate", "up", "down")):
        w = s.w[i]
        t = w.scales if group else w
        keep = t[e].clone()
        t[e] = float("inf")
        s.call(y=y)
        for tok in range(12):
            if e in idx[tok].tolist():
                assert not y[tok].isfinite().all(), (name, tok)
            else:
                assert torch.equal(y[tok], want[tok]), (name, tok)
        t[e] = keep


@kinds
@pytest.mark.parametrize("T,K", [(3, 2), (6, 8), (16, 2)])
def test_infinite_down_weights_keep_their_sign(dtype, group, T, K):
    """An infinity among the down weights makes an output the infinity that the products give, not a NaN: one per row here (4 bits: an
    infinite scale, by which the group's sum is multiplied, of one code that is not 8), so that there is no other to take away from it."""
    s = Layer(T, 256, 8, K, 320 if group < 64 else 384, dtype=dtype, group=group, seed=5)
    want = s.call().clone()
    idx, weight = s.plan.layer_tensor(0).tolist(), s.plan.layer_tensor(1)
    assert (weight > 0).all()
    e, rows = idx[0][0], [0, 7, 130, 255]
    for i, (h, f) in enumerate(zip(rows, (3, 64, 131, 319))):
        value = float("inf") if i % 2 else float("-inf")
        if group:
            s.w[2].scales[e, f // group, h] = value
            q = torch.zeros(group, dtype=torch.int32, device="cuda")
            q[f % group] = 3
            lo = f // group * group // 2
            s.w[2].codes[e, h, lo:lo + group // 2] = R.encode(q.unsqueeze(0))[0]
        else:
            s.w[2][e, h, f] = value
    y = s.call()
    gate, up = s.matrix(0)(e), s.matrix(1)(e)
    for t in range(T):
        if e not in idx[t]:
            assert torch.equal(y[t], want[t])
            continue
        for i, (h, f) in enumerate(zip(rows, (3, 64, 131, 319))):
            g, u = gate[f] @ s.x[t].double(), up[f] @ s.x[t].double()
            sign = torch.sign(g * u) * (1 if i % 2 else -1)   # (silu has its argument's sign)
            assert y[t, h] == sign * float("inf"), (t, h, y[t, h].item())
        rest = [h for h in range(256) if h not in rows]
        assert torch.equal(y[t, rest], want[t, rest])


@kinds
def test_same_bytes_every_time(dtype, group):
    s = Layer(10, 1024, 24, 3, 768, dtype=dtype, group=group)
    first = s.call().clone()
    for _ in range(5):
        s.y.zero_()
        assert torch.equal(s.call(), first)


@kinds
def test_tensor_parallel_shards_change_nothing(dtype, group):
    s = Layer(5, 512, 8, 2, 512, dtype=dtype, group=group, renorm=1)
    first = s.call().clone()
    tp = B.Plan(B.make_config(5, 512, 8, 1, 2, 512, s.plan.cfg.dtype, renormalize=1, tp_shards=4))
    assert torch.equal(s.call(plan=tp, y=torch.empty_like(first)), first)
    idx, w = s.plan.layer_tensor(0), s.plan.layer_tensor(1)
    shards = (idx[..., None] * 4 + torch.arange(4, device="cuda", dtype=torch.int32)).flatten(1)
    assert torch.equal(tp.layer_tensor(0), shards) and torch.equal(tp.layer_tensor(1), w.repeat_interleave(4, 1))
    assert torch.equal(tp.layer_tensor(3), s.plan.layer_tensor(3).repeat_interleave(4))


@pytest.mark.parametrize("mode", range(4))
def test_between_calls_of_the_layer(mode):
    """moe_layer and moe_layer_few take turns on one plan: neither disturbs the other, in any dispatch scheme."""
    s = Layer(12, 512, 16, 2, 256, dispatch_mode=mode)
    want, few = torch.empty_like(s.y), s.call().clone()
    s.plan.moe_layer(s.x, s.wr, s.bias, *s.w, want)
    y = torch.empty_like(s.y)
    for _ in range(3):
        assert torch.equal(s.call(), few)
        s.plan.moe_layer(s.x, s.wr, s.bias, *s.w, y)
        assert torch.equal(y, want) and s.plan.moe_last_status() == (0, 0)


@kinds
def test_captured_and_replayed(dtype, group):
    s = Layer(6, 768, 12, 3, 512, dtype=dtype, group=group)
    want = s.call().clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call()
        s.call()
    x2 = s.x.flip(0).clone()
    for x, y in ((s.x.clone(), want), (x2, want.flip(0))):
        s.x.copy_(x)
        s.y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.y, y)
    s.y.zero_()
    assert torch.equal(s.call(), want.flip(0))


@kinds
def test_two_plans_on_two_streams_at_once(dtype, group):
    """Two calls whose CTAs each wait for one another: a cooperative launch starts whole or not at all."""
    a, b = Layer(4, 2048, 16, 2, 1024, dtype=dtype, group=group, seed=1), Layer(9, 1024, 16, 4, 2048, dtype=dtype, group=group, seed=2)
    wa, wb = a.call().clone(), b.call().clone()
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    a.y.zero_(), b.y.zero_()
    torch.cuda.synchronize()
    for _ in range(50):
        a.call(stream=sa)
        b.call(stream=sb)
    torch.cuda.synchronize()
    assert a.plan.moe_last_status() == (0, 0) and b.plan.moe_last_status() == (0, 0)
    assert torch.equal(a.y, wa) and torch.equal(b.y, wb)


@kinds
def test_beside_a_kernel_that_fills_the_gpu(dtype, group):
    s = Layer(4, 1024, 16, 2, 1024, dtype=dtype, group=group)
    want = s.call().clone()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    other, here = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(other):
        for _ in range(20):
            big @ big
    for _ in range(20):
        s.call(stream=here)
    torch.cuda.synchronize()
    assert s.plan.moe_last_status() == (0, 0) and torch.equal(s.y, want)


@kinds
def test_output_in_the_place_of_the_tokens(dtype, group):
    s = Layer(5, 512, 8, 2, 256, dtype=dtype, group=group)
    want = s.call().clone()
    assert torch.equal(s.call(y=s.x), want)


def test_first_call_of_a_plan_inside_a_capture():
    s = Layer(3, 512, 8, 2, 256, seed=4)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.call()
    graph.replay()
    torch.cuda.synchronize()
    got = s.y.clone()
    assert torch.equal(s.check(), got)


def test_plan_made_behind_other_work_and_first_called_on_a_stream_of_its_own():
    """What plan creation leaves on the device is there before a stream that nothing orders can call."""
    s = Layer(3, 512, 8, 2, 256, seed=4)
    want, here = s.call().clone(), torch.cuda.Stream()
    big = torch.randn(8192, 8192, device="cuda")
    for fill in (0x7f, 0xff):
        size = B.moe_workspace_bytes(s.plan.cfg) + 256
        torch.full((size,), fill, dtype=torch.uint8, device="cuda")  # (freed: the plan's workspace is likely to be the same memory)
        y = torch.zeros_like(s.y)
        torch.cuda.synchronize()
        for _ in range(20):
            big @ big
        plan = B.Plan(s.plan.cfg)
        s.call(y=y, plan=plan, stream=here)
        here.synchronize()
        assert plan.moe_last_status() == (0, 0) and torch.equal(y, want)


def plan_on(room, cfg, nbytes):
    """A plan on given memory (a Plan takes as much as it may), or the library's refusal."""
    plan = B.Plan.__new__(B.Plan)
    plan.cfg, plan.device, plan.P, plan.workspace, plan.handle = cfg, room.device, B.moe_pool_tiles(cfg), room, ctypes.c_void_p()
    rc = B.lib().moe_plan_create(ctypes.byref(cfg), room.data_ptr(), nbytes, ctypes.byref(plan.handle))
    return plan if rc == 0 else rc


@pytest.mark.parametrize("T,dtype", [(1, BF16), (16, BF16), (7, FP32)])
def test_workspace_without_room_for_the_one_launch_layer(T, dtype):
    """A workspace without what this layer alone needs is enough for every other call."""
    s = Layer(T, 264, 8, 2, 136, dtype=dtype)
    want, full = torch.empty_like(s.y), B.moe_workspace_bytes(s.plan.cfg)
    s.plan.moe_layer(s.x, s.wr, None, *s.w, want)
    saved = T * (8 * 264 + 66560) + 512
    lean = full - saved
    room = torch.empty(full, dtype=torch.uint8, device="cuda")
    for nbytes, few in ((lean, False), (full - 1, False), (full, True)):
        room.fill_(0xff)
        plan = plan_on(room, s.plan.cfg, nbytes)
        for _ in range(2):
            s.y.zero_()
            plan.moe_layer(s.x, s.wr, None, *s.w, s.y)
            assert torch.equal(s.y, want) and plan.moe_last_status() == (0, 0)
            if few:
                assert torch.equal(s.call(plan=plan).clone(), s.call())
                continue
            s.y.fill_(7.0)
            with pytest.raises(B.MoeError) as err:
                s.call(plan=plan)
            assert err.value.code == -7 and (s.y == 7.0).all()
        assert (room[nbytes:] == 0xff).all()
        plan.close()
    assert plan_on(room, s.plan.cfg, lean - 256) == -7


def test_plan_creation_waits_for_nothing():
    s = Layer(2, 512, 8, 2, 256)
    room = torch.empty(B.moe_workspace_bytes(s.plan.cfg), dtype=torch.uint8, device="cuda")
    big = torch.randn(8192, 8192, device="cuda")
    big @ big
    done = torch.cuda.Event()
    torch.cuda.synchronize()
    for _ in range(20):
        big @ big
    done.record()
    plan = plan_on(room, s.plan.cfg, room.numel())
    assert not done.query()                               # (a tenth of a second of work)
    y = torch.zeros_like(s.y)
    assert torch.equal(s.call(plan=plan, y=y), s.call())


def test_first_call_captured_and_never_replayed_or_replayed_in_between():
    """Whatever the workspace held, and whichever of a graph and a plain call runs first: both find the barriers' start."""
    s = Layer(4, 512, 8, 2, 256, seed=6)
    want = s.call().clone()
    for fill in (0x7f, 0xff):
        for replays in (0, 1, 3):
            room = torch.full((B.moe_workspace_bytes(s.plan.cfg),), fill, dtype=torch.uint8, device="cuda")
            plan = plan_on(room, s.plan.cfg, room.numel())
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            y = torch.zeros_like(want)
            with torch.cuda.graph(graph):
                s.call(plan=plan, y=y)
                s.call(plan=plan, y=y)
            for _ in range(replays):
                y.zero_()
                graph.replay()
                assert torch.equal(y, want) and plan.moe_last_status() == (0, 0)
            for _ in range(3):
                for run in (lambda: s.call(plan=plan, y=y), lambda: s.call(plan=plan, y=y), graph.replay):
                    y.zero_()
                    run()
                    assert torch.equal(y, want) and plan.moe_last_status() == (0, 0)


def test_gate_results_that_only_fp32_holds():
    """silu(g) u between bf16's largest number and fp32's is not an infinity on the way to a small output."""
    s = Layer(1, 8, 1, 1, 8)
    s.x.zero_()[0, :2] = 1.0
    s.wr.zero_()
    for w in s.w:
        w.zero_()
    s.w[0][0, 0, 0] = 2.0 ** 64
    s.w[1][0, 0, :2] = torch.tensor([2.0 ** 64 * 255 / 256, 2.0 ** 64 * 3 / 1024], device="cuda")
    s.w[2][0, 3, 0] = 2.0 ** -100
    y = s.check()
    assert y[0, 3].item() == 2.0 ** 28 and y.isfinite().all()


def test_wait_that_runs_out_is_reported():
    """A limit of one nanosecond: the barriers give up, the status says so, and the plan's counters are as before."""
    s = Layer(2, 512, 8, 2, 256, wait_limit_ns=1)
    s.call()
    code, detail = s.plan.moe_last_status()
    assert B.strerror(code) == "bounded device-side wait ran out" and detail == 9
    s.call()
    assert s.plan.moe_last_status()[0] == code
    Layer(2, 512, 8, 2, 256).check()


@pytest.mark.parametrize("kw,barriers", [(dict(T=2, H=512, E=8, K=2, F=256), 2), (dict(T=16, H=36, E=16, K=4, F=8192, dtype=FP32), 3)])
def test_barriers_count_right_after_waits_that_ran_out(kw, barriers):
    """Every launch adds 2^31 to each of its barriers' counters, whether or not a wait in it ran out.  Two equal calls leave the same workspace but
    for the counters, which is how they are found."""
    s = Layer(**kw, seed=3)
    words = lambda plan: plan.workspace[:plan.workspace.numel() // 4 * 4].view(torch.int32)  # noqa: E731
    s.call()
    before = words(s.plan).clone()
    s.call()
    at = (words(s.plan) != before).nonzero().flatten()
    assert at.numel() == barriers and (words(s.plan)[at] ^ before[at] == -2 ** 31).all()
    plan = B.Plan(B.make_config(s.T, s.H, s.E, 1, s.K, s.F, s.plan.cfg.dtype, wait_limit_ns=1))
    assert plan.workspace.numel() == s.plan.workspace.numel() and plan.workspace.data_ptr() % 256 == s.plan.workspace.data_ptr() % 256 == 0
    late = 0
    for n in range(1, 9):
        s.call(plan=plan)
        late += plan.moe_last_status() != (0, 0)
        assert (words(plan)[at] == (-2 ** 31 if n % 2 else 0)).all(), n
    assert late > 0


def test_empty_batch():
    plan = B.Plan(B.make_config(0, 64, 4, 1, 2, 64, B.DTYPE_BF16))
    w = torch.zeros(4, 64, 64, dtype=BF16, device="cuda")
    plan.moe_layer_few(None, torch.zeros(4, 64, dtype=BF16, device="cuda"), None, w, w, w, None)
    assert plan.moe_last_launch_count() == 0


@pytest.mark.parametrize("tp", [1, 2])
def test_empty_batch_leaves_no_counts_behind(tp):
    """The rows per expert hold the call's values behind it, also where there are no rows."""
    wr, w = torch.zeros(4, 64, dtype=BF16, device="cuda"), torch.zeros(4, 64, 64, dtype=BF16, device="cuda")
    q = B.W4.empty(64, 64, 32, experts=4)
    plan = B.Plan(B.make_config(0, 64, 4, 1, 2, 64, B.DTYPE_BF16, tp_shards=tp))
    for call in (lambda: plan.moe_layer_few(None, wr, None, w, w, w, None), lambda: plan.moe_layer_few_w4(None, wr, None, q, q, q, None)):
        plan.layer_tensor(3).fill_(55)
        call()
        assert plan.layer_tensor(3).tolist() == [0] * (4 * tp) and plan.moe_last_launch_count() == 0 and plan.moe_last_status() == (0, 0)


def test_calls_refuse_what_they_cannot_take():
    s, q = Layer(4, 128, 4, 2, 64), Layer(4, 128, 4, 2, 64, group=64)

    def code(f, *a):
        with pytest.raises(B.MoeError) as err:
            f(*a)
        return err.value.code

    wide = B.Plan(B.make_config(17, 128, 4, 1, 2, 64, B.DTYPE_BF16))
    x17 = torch.zeros(17, 128, dtype=BF16, device="cuda")
    assert code(wide.moe_layer_few, x17, s.wr, None, *s.w, x17) == -3
    assert code(wide.moe_layer_few_w4, x17, s.wr, None, *q.w, x17) == -3
    ident = B.Plan(B.make_config(4, 128, 4, 1, 2, 0, B.DTYPE_BF16, identity_experts=1))
    assert code(ident.moe_layer_few, s.x, s.wr, None, *s.w, s.y) == -1
    fp32 = B.Plan(B.make_config(4, 128, 4, 1, 2, 64, B.DTYPE_FP32))
    assert code(fp32.moe_layer_few_w4, s.x, s.wr, None, *q.w, s.y) == -3
    for missing in range(7):
        args = [s.x, s.wr, None, *s.w, s.y]
        if missing == 2:
            continue
        args[missing] = None
        assert code(s.plan.moe_layer_few, *args) == -1, missing
        args = [s.x, s.wr, None, *s.w, s.y]
        args[missing] = args[missing].data_ptr() + 8
        assert code(s.plan.moe_layer_few, *args) == -2, missing
    assert code(s.plan.moe_layer_few, s.x, s.wr, torch.zeros(4, device="cuda").data_ptr() + 2, *s.w, s.y) == -2
    other = Layer(4, 128, 4, 2, 64, group=32)
    with pytest.raises(ValueError):
        s.plan.moe_layer_few_w4(s.x, s.wr, None, q.w[0], other.w[1], q.w[2], s.y)
    with pytest.raises(ValueError):
        s.plan.moe_layer_few_w4(s.x, s.wr, None, q.w[0], q.w[1], q.w[0], s.y)


def test_weights_beyond_four_gigabytes():
    E, H, F = 40, 8192, 8192
    w = [torch.empty(E, F, H, dtype=BF16, device="cuda").normal_(0.0, 0.02) for _ in range(2)]
    w.append(w[0].view(E, H, F))
    s = Layer(2, 8, E, 2, 8)
    s.H, s.F, s.w = H, F, w
    s.x = torch.randn(2, H, device="cuda", dtype=BF16)
    s.wr = torch.randn(E, H, device="cuda").mul_(0.02).to(BF16)
    s.bias = torch.full((E,), float("-inf"), device="cuda")
    s.bias[[0, 36, 39]] = 0.0                   # more than 2^32 bytes apart
    s.plan = B.Plan(B.make_config(2, H, E, 1, 2, F, B.DTYPE_BF16))
    s.room = torch.full((2 * H + 64,), 55.0, dtype=BF16, device="cuda")
    s.y = s.room[:2 * H].view(2, H)
    s.check()


@pytest.mark.parametrize("group", [32, 64, 128])
def test_prefill_and_decoding_on_the_same_4bit_experts(group):
    """As a user has it: dense experts are packed once; a prompt goes through moe_layer on the unpacked weights, the tokens after it
    through the one-launch layer on the codes; a shared expert's projection beside it is a product of its own."""
    H, E, K, F, T = 512, 16, 2, 384, 200
    g = torch.Generator(device="cuda").manual_seed(9)

    def normal(std, *shape):
        return torch.empty(shape, dtype=BF16, device="cuda").normal_(0.0, std, generator=g)

    dense = [normal(0.05, E, F, H), normal(0.05, E, F, H), normal(0.05, E, H, F)]
    wr, x = normal(0.05, E, H), normal(1.0, T, H)
    packed, back = [], []
    for w in dense:
        packed.append(B.W4.empty(w.shape[1], w.shape[2], group, experts=E))
        B.moe_w4_pack(w, packed[-1])
        back.append(torch.empty_like(w))
        B.moe_w4_unpack(packed[-1], back[-1])
        # the form's own error: half a step of the scale at most, and what the scale's and the weight's rounding to bf16 add
        step = packed[-1].scales.double().transpose(1, 2).repeat_interleave(group, dim=2)
        assert ((back[-1].double() - w.double()).abs() <= step * (0.5 + 7 * 2.0 ** -8) + 2.0 ** -8 * w.double().abs()).all()
    prompt, y = B.Plan(B.make_config(T, H, E, 1, K, F, B.DTYPE_BF16)), torch.empty_like(x)
    prompt.moe_layer(x, wr, None, *back, y)
    shared = B.W4(packed[0].codes[3], packed[0].scales[3])
    for T1 in (1, 5, 16):
        plan = B.Plan(B.make_config(T1, H, E, 1, K, F, B.DTYPE_BF16))
        few, proj = torch.empty(T1, H, dtype=BF16, device="cuda"), torch.empty(T1, F, dtype=BF16, device="cuda")
        for t0 in range(0, 48, T1):
            rows = x[t0:t0 + T1]
            if rows.shape[0] < T1:
                break
            plan.moe_layer_few_w4(rows, wr, None, *packed, few)
            B.moe_w4_matvec(shared, rows, None, proj)
            # the definition on the unrounded 4-bit weights
            idx = plan.layer_tensor(0).long()
            m = [lambda e, w=w: R.weights(w.codes[e], w.scales[e]) for w in packed]
            logits, dl, _, want, bound = R.layer(rows.double(), wr.double(), None, *m, K, 0, idx, BF16)
            R.check_picks(idx, logits, dl)
            R.assert_within(few, want, bound, "decoded tokens")
            p, pb = R.matvec(R.weights(shared.codes, shared.scales), rows.double())
            R.assert_within(proj, p, pb + R.HALF[BF16] * (p.abs() + pb), "projection")
            # and the prompt's rows are the same tokens on weights rounded to bf16
            assert torch.equal(idx, prompt.layer_tensor(0)[t0:t0 + T1].long())
            diff = (few.double() - y[t0:t0 + T1].double()).norm() / y[t0:t0 + T1].double().norm()
            assert diff < 2e-2  # (three roundings of the weights and two of what is stored, each 2^-8 of a value at most)
