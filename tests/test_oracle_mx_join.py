"""The plain forms of the 4-bit operators and of the residual joint: the format
against its definition value by value, the gradients against differences."""
import numpy as np
import pytest

from oracle import join_ref, mx_ref


def test_codes_of_known_values():
    x = np.zeros((1, 32))
    x[0, :12] = [6, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -1.5, 4]
    codes, scales = mx_ref.quantize(x)
    assert scales[0, 0] == 127  # top 6 = 1.5 x 2^2: e = 0
    c = np.stack((codes & 15, codes >> 4), 2).reshape(-1)[:12]
    assert c.tolist() == [7, 0, 1, 2, 2, 4, 4, 6, 6, 7, 8 + 3, 6]
    v = mx_ref.values(codes, scales, 12)
    assert v[0].tolist() == [6, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, -1.5, 4]


def test_saturates_and_scales():
    x = np.zeros((4, 40))
    x[0, 0] = 7.9  # above 6 at e = 0
    x[1, 0] = 8.0  # e = 1
    x[2, 33] = 2.0 ** -140  # e at its least: 2^-13 of the unit
    codes, scales = mx_ref.quantize(x)
    v = mx_ref.values(codes, scales, 40)
    assert v[0, 0] == 6.0 and scales[0, 0] == 127
    assert v[1, 0] == 8.0 and scales[1, 0] == 128
    assert scales[2, 1] == 0 and v[2, 33] == 0.0
    assert (scales[3] == 0).all() and not codes[3].any()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_non_finite_block(bad):
    x = np.ones((1, 64))
    x[0, 40] = bad
    codes, scales = mx_ref.quantize(x)
    v = mx_ref.values(codes, scales, 64)
    assert scales[0].tolist() == [125, 255] and (v[0, :32] == 1).all() and np.isnan(v[0, 32:]).all()


def test_rounds_to_the_nearest_level():
    r = np.random.default_rng(3)
    x = r.normal(size=(50, 96)) * np.exp2(r.integers(-20, 20, size=(50, 1)))
    codes, scales = mx_ref.quantize(x)
    unit = np.repeat(np.exp2(scales.astype(float) - 127), 32, axis=1)
    levels = np.concatenate((mx_ref.LEVELS, -mx_ref.LEVELS))
    best = np.abs(x[:, :, None] / unit[:, :, None] - levels).min(axis=2) * unit
    got = np.abs(mx_ref.values(codes, scales, 96) - x)
    assert (got == best).all()
    assert (np.abs(x / unit) < 8).all() and (np.abs(x / unit).reshape(50, 3, 32).max(axis=2) >= 4).all()


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("groups", [0, 1, 3, 6])
def test_joint_gradients_against_differences(kind, post, groups):
    r = np.random.default_rng(5)
    rows, cols = 6, 11
    t = {"x": r.normal(size=(rows, cols)), "y": r.normal(size=(rows, cols)), "w1": r.normal(size=cols),
         "b1": r.normal(size=cols), "w2": r.normal(size=cols), "b2": r.normal(size=cols)}
    if not post:
        t["w1"] = t["b1"] = None
    t["gate"] = r.normal(size=(groups, cols)) if groups else None
    dr, dn = r.normal(size=(rows, cols)), r.normal(size=(rows, cols))

    def loss(**k):
        a = dict(t, **k)
        f = join_ref.forward(a["x"], a["y"], kind, post, a["w1"], a["b1"], a["gate"], 0.7, a["w2"], a["b2"], 1e-3)
        return (f["r"] * dr).sum() + (f["n"] * dn).sum()

    g = join_ref.backward(dr, dn, t["x"], t["y"], kind, post, t["w1"], t["b1"], t["gate"], 0.7, t["w2"], 1e-3)
    for name, v in t.items():
        if v is None:
            continue
        u = r.normal(size=v.shape)
        d = (loss(**{name: v + 1e-6 * u}) - loss(**{name: v - 1e-6 * u})) / 2e-6
        assert abs((g["d" + name] * u).sum() - d) <= 1e-6 * (1 + abs(d)), name
