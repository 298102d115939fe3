"""The quantised act step behind bf16 conv layers, level by level: with one tap of a power of two per channel, pixels 0 and 255 and short biases every value of the conv layers
has at most eight significant bits, so bf16 holds it exactly and what follows has to be the oracle's but for fp32's own rounding."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2111_01264_amd as P
from datagen import synth
from oracle import actor
from tests.gpu_util import blob_slices, dev, make_cfg
from tests.test_gpu_act_sampled import Out, features, near_border


def exact_conv_params(A, seed):
    """The fully connected layers as ever; conv layers of single taps."""
    r = np.random.default_rng(seed)
    theta, s = synth.init_params(seed, A).copy(), blob_slices(A)
    for name, (o, c, k), taps, step in (("conv1", (32, 4, 8), [0.5, 1.0], 0.25), ("conv2", (64, 32, 4), [0.5, 1.0, -0.5], 0.25), ("conv3", (64, 64, 3), [0.5, 1.0, -1.0], 0.125)):
        w = np.zeros((o, c, k, k), np.float32)
        w[np.arange(o), r.integers(0, c, o), r.integers(0, k, o), r.integers(0, k, o)] = r.choice(taps, o)
        theta[s[name + ".w"]] = w.ravel()
        theta[s[name + ".b"]] = r.integers(0, 4, o) * step
    return theta


def quantised_rows(theta, x, A):
    """Q rows from features that are exact, and how far off they may be: a hidden value one step of fp32 off (its fp64 arithmetic in another order, at a border of fp32) moves a level
    that lies within that of its own border; the scale's, the product's and the result's roundings."""
    s = blob_slices(A)
    levels = {}
    for name, shape in (("fc1", (512, 3136)), ("fc2", (A, 512))):
        q, sc = actor.quantize_rows(theta[s[name + ".w"]].reshape(shape).astype(np.float64))
        levels[name] = q, sc.astype(np.float32).astype(np.float64), theta[s[name + ".b"]].astype(np.float64)
    fl32 = lambda v: v.astype(np.float32).astype(np.float64)  # noqa: E731
    xq, sx = actor.quantize_rows(x)
    h = fl32(actor.linear(xq, fl32(sx), *levels["fc1"], relu=True))
    hq, sh = actor.quantize_rows(h)
    w2, s2, b2 = levels["fc2"]
    q = actor.linear(hq, fl32(sh), w2, s2, b2)
    top = h.max(1, keepdims=True)
    moved = near_border(h, top, 2.0 ** -22 * top).astype(np.float64)
    off = sh[:, None] * (moved @ np.abs(w2).T) * s2 + 2.0 ** -22 * actor.linear(np.abs(hq), sh, np.abs(w2), s2) + 2.0 ** -24 * np.abs(q)
    return q, off, hq


@pytest.mark.parametrize("A,W", [(1, 1), (18, 8), (18, 40), (32, 130)])
def test_quantised_rows_behind_exact_features(A, W):
    sa, st = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = P.dqn_create(make_cfg(A, max_envs=W, precision=P.DQN_PRECISION_BF16, seed=3), sa, st)
    try:
        thetas = exact_conv_params(A, 50), exact_conv_params(A, 51)
        P.dqn_set_params(ctx, P.DQN_PARAMS_ONLINE, thetas[0])
        P.dqn_set_params(ctx, P.DQN_PARAMS_TARGET, thetas[1])
        states = np.where(np.random.default_rng(W).random((W, 4, 84, 84)) < 0.5, 255, 0).astype(np.uint8)
        for use_target in (1, 0):
            x = features(thetas[use_target], states, A)
            assert np.array_equal(torch.as_tensor(x).bfloat16().double().numpy(), x) and len(np.unique(x, axis=0)) == W
            want, off, hq = quantised_rows(thetas[use_target], x, A)
            assert np.all(np.count_nonzero(hq, axis=1) > 50) and off.max() < 0.02 * np.abs(want).max()   # (a row off by a level or two is seen)
            P.dqn_quantize_actor(ctx, use_target)
            out = Out(W, A)
            P.dqn_act_sampled(ctx, dev(states), W, None, None, None, None, None, 5, use_target, 1, out.actions[:W], out.q, out.logp[:W])
            q = out.read()[1]
            assert np.all(np.abs(q - want) <= off), (np.abs(q - want).max(), off.max())
    finally:
        P.dqn_destroy(ctx)
