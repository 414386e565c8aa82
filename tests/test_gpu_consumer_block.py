"""The whole layer of the LLM task over placed embeddings: its calls as they follow one another, in prompts and recorded steps, every
stage against the CPU oracle on what the stage before gave."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2603_12118_amd import binding as B
from paper_2603_12118_amd.consumer_layer import ConsumerBlock, DecodeStep, prompt_positions
from tests.test_gpu_block import host, within

pytestmark = pytest.mark.gpu


def small(**kw):
    d = dict(hidden=256, n_heads=4, n_kv_heads=2, head_dim=64, sections=(8, 12, 12), inter=96, experts=12, top=3, n_pages=32, page_tokens=32, sequences=3,
             max_keys=160, max_position=400)
    return ConsumerBlock(**{**d, **kw})


def values(packed):
    return host(B.cs_weights_read(packed, torch.float32))


def check(block, stages=None):
    s = block.stages if stages is None else stages
    scale = {k: float(np.float32(v)) for k, v in block.scales.items()}
    _, y, _, d = O.norm_residual(host(s["x"]), host(s["x"]), host(block.attention_gain), block_scale=0.0)
    within(s["y"], y, d, "input norm")
    r, z, dr, dz = O.norm_residual(host(s["a"]), host(s["x"]), host(block.expert_gain), post_gain=host(block.post_gains[0]), **scale)
    within(s["r"], r, dr, "stream behind the attention")
    within(s["z"], z, dz, "experts' input")
    m, experts, weights, d = O.moe(host(s["z"]), host(block.router), values(block.up), values(block.down), block.top, score=block.score,
                                   choice_bias=host(block.choice_bias), live=s["live"].cpu().numpy())
    assert np.array_equal(s["experts"].cpu().numpy(), experts)
    within(s["weights"], weights, 2.0 ** -24 * np.abs(weights) * 1.001, "weights")
    within(s["m"], m, d, "experts")
    out, following, do, df = O.norm_residual(host(s["m"]), host(s["r"]), host(block.next_gain), post_gain=host(block.post_gains[1]), **scale)
    within(s["out"], out, do, "stream behind the layer")
    within(s["next"], following, df, "the next layer's input")


def rows(n, hidden=256, seed=0):
    return torch.randn(n, hidden, generator=torch.Generator("cuda:0").manual_seed(seed), device="cuda:0", dtype=torch.bfloat16)


@pytest.mark.parametrize("kw", [dict(), dict(post_norms=False, score="softmax", shared=0, block_scale=0.3), dict(format="bf16", residual_scale=0.9, shared=2)])
def test_prompts_and_recorded_steps(kw):
    block = small(**kw)
    positions, following = prompt_positions([5, (1, 4, 6), 9])
    pos = torch.as_tensor(positions, device="cuda:0")
    block.prefill([0, 2], [rows(38, seed=1), rows(38, seed=2)], [pos, pos])
    check(block)
    block.prefill([1], [rows(1, seed=3)], [pos[:1]])
    check(block)
    step = DecodeStep(block, [following, 1, following])
    stages = dict(block.stages)                              # the recording's tensors
    for i in range(4):
        step.x.copy_(rows(3, seed=10 + i))
        torch.cuda.synchronize()
        step.run()
        torch.cuda.synchronize()
        assert torch.equal(step.out, stages["out"])
        check(block, stages)
        # an eager call between the replays uses tensors of its own
        block.prefill([1], [rows(2, seed=20 + i)], [pos[:2]])
        step.take(1, 2)
    assert block.err.item() == 0


def test_a_sequence_that_is_left_out_goes_through_no_expert():
    block = small()
    pos = torch.as_tensor(prompt_positions([6])[0], device="cuda:0")
    block.prefill([0, 1, 2], [rows(6, seed=i) for i in range(3)], [pos] * 3)
    step = DecodeStep(block, [6, 6, 6])
    stages = dict(block.stages)
    for i in range(3):
        if i == 1:
            block.pages.release(1)
        if i == 2:
            step.take(0, None)
        step.x.copy_(rows(3, seed=30 + i))
        step.x[1] = float("nan") if i else 0.5
        torch.cuda.synchronize()
        step.run()
        torch.cuda.synchronize()
        live = [0, 2] if i == 1 else [2] if i == 2 else [0, 1, 2]
        dead = [b for b in range(3) if b not in live]
        assert (stages["experts"][dead] == -1).all() and not stages["m"][dead].any() and (stages["experts"][live] >= 0).all()
        check(block, {k: v[live] for k, v in stages.items()})


def test_prompts_in_chunks():
    block = small(sequences=2)
    pos = torch.as_tensor(prompt_positions([120])[0], device="cuda:0")
    x = rows(120, seed=5)
    for which, ends in ((0, [120]), (1, [50, 51, 90, 120])):
        for first, last in zip([0] + ends, ends):
            block.prefill([which], [x[first:last]], [pos[first:last]])
            check(block)
    assert block.pages.lens == [120, 120] and block.err.item() == 0


@pytest.mark.parametrize("kw", [dict(), dict(post_norms=False, score="softmax", shared=0), dict(format="bf16", residual_scale=0.9, shared=2)])
def test_rows_of_a_sequence_that_is_left_out_are_zeros_until_take(kw):
    # whatever stands in its row of x
    block = small(**kw)
    pos = torch.as_tensor(prompt_positions([6])[0], device="cuda:0")
    block.prefill([0, 1, 2], [rows(6, seed=i) for i in range(3)], [pos] * 3)
    step = DecodeStep(block, [6, 6, 6])
    stages = dict(block.stages)
    block.pages.release(1)
    for i, left in enumerate((0.5, float("nan"), float("inf"), -3e38)):
        step.x.copy_(rows(3, seed=50 + i))
        step.x[1] = left
        kept = step.x.clone()
        torch.cuda.synchronize()
        step.run()
        torch.cuda.synchronize()
        for name in ("y", "a", "r", "z", "m", "out", "next"):
            assert not stages[name][1].any(), (name, left)               # (a NaN is not zero either)
            assert stages[name][[0, 2]].any(-1).all(), name
        assert not step.out[1].any() and not step.attended[1].any() and step.out.isfinite().all()
        check(block, {k: v[[0, 2]] for k, v in stages.items()})
        assert torch.equal(step.x.view(torch.int16), kept.view(torch.int16))      # the caller's rows are left as they are
    block.prefill([1], [rows(4, seed=60)], [pos[:4]])
    step.take(1, 4)
    step.x.copy_(rows(3, seed=61))
    torch.cuda.synchronize()
    step.run()
    torch.cuda.synchronize()
    assert step.out.any(-1).all()
    check(block, stages)


def test_an_infinity_in_the_stream_is_normed_as_one():
    block = small()
    pos = torch.as_tensor(prompt_positions([5])[0], device="cuda:0")
    x = rows(5, seed=7)
    x[1, 3], x[3, 250] = float("inf"), -float("inf")
    block.prefill([0], [x], [pos])
    y = host(block.stages["y"])
    # 1 / sqrt(mean) is zero: a zero for every finite value, a NaN for the infinity
    with np.errstate(invalid="ignore"):
        want = O.norm(host(x), "rms", host(block.attention_gain), None, 1e-6)[0]
    assert np.isnan(want[1, 3]) and np.isnan(want[3, 250]) and np.isnan(want).sum() == 2
    assert np.array_equal(np.isnan(y), np.isnan(want)) and not y[1, :3].any() and not y[1, 4:].any() and not y[3, :250].any()
