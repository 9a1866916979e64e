"""Pins of the 64-bit activation oracle: hand-worked blocks, nearest codes by going through all of them, gradients by differences."""
import numpy as np
import pytest

import oracle.activations as A


def test_code_values_of_both_formats():
    i8, f8 = A.code_values(A.I8), A.code_values(A.F8)
    assert i8[0] == 0 and i8[1] == 1 / 64 and i8[127] == 127 / 64 and i8[129] == -127 / 64 and i8[255] == -1 / 64 and np.isnan(i8[128])
    assert f8[0x38] == 1.0 and f8[0x7E] == 448 and f8[0xFE] == -448 and f8[0x01] == 2.0 ** -9 and f8[0x08] == 2.0 ** -6
    assert np.isnan(f8[0x7F]) and np.isnan(f8[0xFF])
    torch = pytest.importorskip("torch")
    theirs = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(theirs, f8, equal_nan=True)


@pytest.mark.parametrize("fmt,x,s,codes", [
    (A.I8, [1.0, -0.5, 1 / 128, 3 / 128, 0.0], 127, [64, 224, 0, 2, 0]),            # ties to even
    (A.I8, [127.49 / 64, -127.49 / 64], 127, [127, 129]),                           # just below the tie: still scale 1
    (A.I8, [127.5 / 64, 1 / 64], 128, [64, 0]),                                      # the tie would round to 128: one scale up
    (A.F8, [448.0, -464.0, 1.0], 127, [0x7E, 0xFE, 0x38]),                           # 464 is a tie and rounds down to 448
    (A.F8, [464.01, 2.0], 128, [0x77, 0x38]),                                        # above: 232.005 rounds to 240 under the next scale
    (A.F8, [256.0, 2.0 ** -10, 2.0 ** -10 * 1.5, 2.0 ** -9], 127, [0x78, 0, 1, 1]),  # subnormals, a tie to even
    (A.I8, [0.0, -0.0], 0, [0, 0]),
])
def test_hand_worked_blocks(fmt, x, s, codes):
    q, scale = A.encode(np.array([x]), fmt)
    assert scale[0, 0] == s and q[0].tolist() == codes


@pytest.mark.parametrize("fmt", [A.I8, A.F8])
def test_codes_are_nearest_and_scales_smallest(fmt):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((40, 70)) * np.exp2(rng.integers(-30, 30, (40, 1)))
    x[3] = 0
    x[4, 5], x[5, 40], x[6, 69] = np.inf, np.nan, -np.inf
    q, scale = A.encode(x, fmt)
    assert scale[4].tolist()[0] == 255 and scale[5, 1] == 255 and scale[6, 2] == 255 and np.sum(scale == 255) == 3
    got = A.decode(q, scale, fmt)
    values = A.code_values(fmt)
    values = values[~np.isnan(values)]
    for r in range(x.shape[0]):
        for c in range(x.shape[1]):
            s = scale[r, c // 32]
            if s == 255:
                assert np.isnan(got[r, c])
                continue
            u = 2.0 ** (float(s) - 127)
            assert abs(got[r, c] - x[r, c]) == np.min(np.abs(values * u - x[r, c]))
        for b in range(scale.shape[1]):
            if scale[r, b] in (0, 255):
                continue
            top = np.max(np.abs(x[r, 32 * b:32 * b + 32])) / 2.0 ** (float(scale[r, b]) - 128)   # one scale lower
            assert top >= (127.5 / 64 if fmt == A.I8 else 464)


@pytest.mark.parametrize("pre", [A.NONE, A.RMS, A.LAYER])
@pytest.mark.parametrize("post,gate_kind", [(A.NONE, A.NO_GATE), (A.RMS, A.CHANNEL), (A.LAYER, A.TOKEN), (A.LAYER, A.FULL)])
def test_join_gradients_against_differences(pre, post, gate_kind):
    rng = np.random.default_rng(pre * 8 + post * 2 + gate_kind)
    rows, cols = 5, 9
    p = {"x": rng.standard_normal((rows, cols)), "branch": rng.standard_normal((rows, cols)),
         "w1": rng.standard_normal(cols), "b1": rng.standard_normal(cols), "w2": rng.standard_normal(cols), "b2": rng.standard_normal(cols)}
    shape = {A.NO_GATE: None, A.CHANNEL: (1, cols), A.TOKEN: (rows, 1), A.FULL: (rows, cols)}[gate_kind]
    p["gate"] = rng.standard_normal(shape) if shape else np.ones(())
    dn, dy = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))

    def run(p):
        return A.join_forward(p["x"], p["branch"], 1.3, p["gate"], (pre, 1e-3, p["w1"], p["b1"]), (post, 1e-3, p["w2"], p["b2"]))

    def loss(p):
        y, n = run(p)[:2]
        return (y * dy).sum() + (n * dn).sum()

    _, _, h1, r1, h2, r2 = run(p)
    g = A.join_backward(dn, dy, 1.3, p["gate"], gate_kind, (pre, 1e-3, p["w1"], p["b1"]), (post, 1e-3, p["w2"], p["b2"]), h1, r1, h2, r2)
    names = {"x": "dx", "branch": "dbranch", "w1": "dpre_weight", "b1": "dpre_bias", "w2": "dpost_weight", "b2": "dpost_bias"}
    if shape:
        names["gate"] = "dgate"
    for name, grad in names.items():
        want = np.zeros_like(p[name])
        for i in np.ndindex(p[name].shape):
            hi, lo = ({k: v.copy() for k, v in p.items()} for _ in range(2))
            hi[name][i] += 1e-5
            lo[name][i] -= 1e-5
            want[i] = (loss(hi) - loss(lo)) / 2e-5
        # central differences: h^2 times a third derivative of order 10, and 1e-16 of a loss of order 100 over 2 h
        assert np.allclose(g[grad], want, rtol=1e-6, atol=1e-7), name


def test_weight_gradient_against_differences_and_groups():
    rng = np.random.default_rng(11)
    t, o, k = 7, 4, 5
    kept, dy, w, b = rng.standard_normal((t, k)), rng.standard_normal((t, o)), rng.standard_normal(k), rng.standard_normal(k)
    W, c = rng.standard_normal((o, k)), rng.standard_normal(o)
    dw, db = A.weight_grad(dy, kept, w, b)
    loss = lambda W, c: (((kept * w + b) @ W.T + c) * dy).sum()
    for i in np.ndindex(W.shape):
        d = np.zeros_like(W)
        d[i] = 1e-6
        assert abs((loss(W + d, c) - loss(W - d, c)) / 2e-6 - dw[i]) < 1e-7
    for i in range(o):
        d = np.zeros_like(c)
        d[i] = 1e-6
        assert abs((loss(W, c + d) - loss(W, c - d)) / 2e-6 - db[i]) < 1e-7
    parts, sums = A.weight_grad(dy, kept, w, b, [0, 3, 3, 7])
    assert np.allclose(parts.sum(0), dw) and np.all(parts[1] == 0) and np.allclose(sums.sum(0), db)
    parts, _ = A.weight_grad(dy, kept, w, b, [-4, 2, 1, 90])       # clipped, and a group that would end before it starts
    assert np.allclose(parts[0], A.weight_grad(dy[:2], kept[:2], w, b)[0]) and np.all(parts[1] == 0)
    assert np.allclose(parts[2], A.weight_grad(dy[1:], kept[1:], w, b)[0])
