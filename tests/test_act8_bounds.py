"""How far a value of the 8-bit store may be off (no GPU needed): half a step, which is at most 1 / 127.5 of
its group's largest where the step is not clamped."""
import numpy as np

import ops_ref as R


def _errors(x):
    """|stored - x|, the half steps and the groups' largest, float64 [rows, 32]."""
    x = np.asarray(x, np.float64)
    _, E, val = R.act8_ref(x)
    return np.abs(val - x), np.ldexp(0.5, E.astype(int) - 133), np.abs(x).max(1, keepdims=True), E


def test_border_where_the_step_doubles():
    """A largest of 127.5 old steps takes the doubled step: 63.75 of them, rounded to 64 (ties to even)."""
    x = np.zeros((1, 32))
    x[0, 0], x[0, 1] = 127.5 / 64, 0.5 / 32
    err, half, top, E = _errors(x)
    assert E[0, 0] == 128 and err[0, 1] == half[0, 0] == 1 / 64
    assert err[0, 1] / top[0, 0] == 1 / 127.5 > 2.0 ** -7
    x[0, 0] = np.nextafter(np.float32(127.5 / 64), np.float32(0))  # just below: half the step
    assert _errors(x)[3][0, 0] == 127


def test_errors_of_many_groups():
    r = np.random.default_rng(0)
    x = (r.uniform(-1, 1, (20000, 32)) * np.exp2(r.uniform(-100, 100, (20000, 1)))).astype(np.float32)
    err, half, top, E = _errors(x)
    assert (E > 7).all() and (E < 254).all()
    assert (err <= half).all() and (err <= top / 127.5).all()


def test_clamped_steps():
    """Below, half a step of 2^-126 is all that holds; above, values past 127.5 steps of 2^121 end at 127."""
    x = np.zeros((2, 32))
    x[0, :3] = 2.0 ** -126, 2.0 ** -127, 1.5 * 2.0 ** -127
    x[1, :2] = np.finfo(np.float32).max, 2.0 ** 120
    err, half, top, E = _errors(x)
    assert E[0, 0] == 7 and E[1, 0] == 254
    assert (err[0] <= half[0]).all() and err[0, 1] == top[0, 0] / 2
    assert half[1, 0] < err[1, 0] < 2 * half[1, 0] and err[1, 1] <= half[1, 0]
