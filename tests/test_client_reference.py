"""The 64-bit forms the client's kernels are compared with, checked on their
own (CPU): Philox against its published known answers, the residual norm's
gradients against central differences, the 8-bit rounding against torch's."""
import numpy as np
import pytest

import client_reference as ref


@pytest.mark.parametrize("counter, seed, want", [
    ((0, 0, 0, 0), 0, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, 0xFFFFFFFFFFFFFFFF, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
])
def test_philox_known_answers(counter, seed, want):
    got = ref.philox4x32_10(*[np.array([c]) for c in counter], seed)
    assert tuple(int(w[0]) for w in got) == want


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", [None, "channel", "row", "full"])
@pytest.mark.parametrize("act", ["identity", "sigmoid", "tanh"])
@pytest.mark.parametrize("post, pre", [(True, True), (False, True), (True, False), (False, False)])
def test_residual_norm_gradients_match_differences(layer, gate, act, post, pre):
    rng = np.random.default_rng(5)
    r, c, rho, eps = 3, 7, 0.7, 1e-3
    m = ref.drop_factor(r, c, (0.3, 99, 5, 2, 1))
    x = {"branch": rng.normal(size=(r, c)), "residual": rng.normal(size=(r, c))}
    for name, there in (("w_post", post), ("b_post", post), ("w_pre", pre), ("b_pre", pre)):
        x[name] = rng.normal(size=c) if there else None
    x["gate"] = {None: None, "channel": rng.normal(size=c), "row": rng.normal(size=(r, 1)),
                 "full": rng.normal(size=(r, c))}[gate]
    ks, kh = rng.normal(size=(r, c)), rng.normal(size=(r, c))

    def loss(x):
        s = ref.residual_norm_sum(x["branch"], x["residual"], layer, x["w_post"], x["b_post"], x["gate"], act, rho,
                                  eps, m)
        out = (s * ks).sum()
        return out + (ref.residual_norm_normed(s, layer, x["w_pre"], x["b_pre"], eps) * kh).sum() if pre else out

    total = ref.residual_norm_sum(x["branch"], x["residual"], layer, x["w_post"], x["b_post"], x["gate"], act, rho,
                                  eps, m)
    g = ref.residual_norm_backward(x["branch"], total, ks, kh if pre else None, layer, x["w_post"], x["b_post"],
                                   x["w_pre"], x["b_pre"], x["gate"], act, rho, eps, m)
    h = 1e-5
    for name, v in x.items():
        if v is None:
            continue
        want = np.zeros_like(v)
        for i in np.ndindex(v.shape):
            up, down = dict(x), dict(x)
            up[name], down[name] = v.copy(), v.copy()
            up[name][i] += h
            down[name][i] -= h
            want[i] = (loss(up) - loss(down)) / (2 * h)
        # central differences: h^2 times a third derivative (eps 1e-3 bounds rstd by 32) and 1e-16 / h of rounding
        np.testing.assert_allclose(g["d" + name], want, rtol=1e-5, atol=1e-6, err_msg=name)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_8bit_rounding_matches_torch(fmt):
    import torch
    rng = np.random.default_rng(6)
    y = np.concatenate([rng.normal(size=20000) * np.exp2(rng.uniform(-18, 6, size=20000)),
                        ref.FMAX[fmt] * np.linspace(-1, 1, 4001), [0.0, -0.0]]).astype(np.float32)
    y = y[np.abs(y) <= ref.FMAX[fmt]]
    want = torch.from_numpy(y).to(torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2).double().numpy()
    np.testing.assert_array_equal(ref.round_8bit(y.astype(np.float64), fmt), want)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_block_exponent_is_the_smallest(fmt):
    f = ref.FMAX[fmt]
    amax = np.array([f, np.nextafter(f, 1e9), f * 2, f / 2, 1.0, 1e-30, 3.4e38, f * 2.0 ** -126, f * 2.0 ** -127, 1e-45])
    e = ref.block_exponent(amax, fmt)
    assert np.all(amax <= f * np.exp2(e.astype(float)))
    assert np.all((e == -126) | (amax > f * np.exp2(e.astype(float) - 1)))
    assert ref.block_exponent(np.array([0.0]), fmt)[0] == 0
