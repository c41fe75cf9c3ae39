"""The 64-bit reference of attention with heads, bias and dropout against known answers and differences, and the tables of buckets."""
import math

import numpy as np
import pytest

from heads_ref import Attention, bucket_of, keep_factors, threefry


def test_threefry_known_answers():
    """The published vectors of the 20-round form."""
    F = 0xFFFFFFFF
    assert threefry((0, 0), 0, 0, 20) == (0x6B200159, 0x99BA4EFE)
    assert threefry((F, F), F, F, 20) == (0x1CB996FC, 0xBB002BE7)
    assert threefry((0x13198A2E, 0x03707344), 0x243F6A88, 0x85A308D3, 20) == (0xC4923A9C, 0x483DF7A0)


def test_dropout_keeps_the_right_share_and_differs_by_head_step_and_seed():
    z = keep_factors(3, 200, 300, 0.3, (7, 1))
    assert abs((z > 0).mean() - 0.7) < 5 * math.sqrt(0.21 / z.size)
    other = [keep_factors(3, 200, 300, 0.3, s) for s in ((8, 1), (7, 2), (7 + (1 << 40), 1))]
    for a in other + [z[[1, 2, 0]]]:
        assert abs(((a > 0) == (z > 0)).mean() - 0.58) < 0.01  # independent: .7^2 + .3^2


def _problem(rng, heads=2, kv=1):
    M, K, d, N = 6, 9, 8, 8
    stored = rng.random((M, K)) < 0.5
    stored[2] = False
    return dict(stored=stored, X=rng.standard_normal((M, heads, d)), Y=rng.standard_normal((K, kv, d)), H=rng.standard_normal((K, kv, N)), scale=0.3,
                table=rng.standard_normal((heads, 5)), buckets=[0, 1, 2, 2, 3, 4, 7], shift=1, p=0.4, state=(5, 3))


@pytest.mark.parametrize("name", ["X", "Y", "H", "table"])
def test_gradients_of_the_reference_against_differences(name):
    rng = np.random.default_rng(3)
    a = _problem(rng)
    G = rng.standard_normal((6, 2, 8))
    ref = Attention(**a)
    out, lse, _, _ = ref.forward()
    assert np.isneginf(lse[:, 2]).all() and not out[2].any()
    g, _ = ref.backward(out, lse, G)
    got = g["dTable" if name == "table" else "d" + name]
    for at in [tuple(rng.integers(0, n) for n in a[name].shape) for _ in range(12)]:
        h, side = 1e-5, []
        for sign in (1, -1):
            moved = a[name].copy()
            moved[at] += sign * h
            side.append((Attention(**{**a, name: moved}).forward()[0] * G).sum())
        assert abs((side[0] - side[1]) / (2 * h) - got[at]) < 1e-7 * max(1, abs(got[at]))


@pytest.mark.parametrize("buckets,distance,both", [(32, 128, True), (32, 128, False), (8, 16, True), (12, 1000, True), (64, 40, True), (5, 9, False), (2, 2, False)])
def test_relative_buckets(buckets, distance, both):
    import paper_2412_11007_amd as fs
    table = fs.fs_relative_buckets(buckets, distance, both, device="cpu").tolist()
    assert len(table) == 2 * distance + 1
    n = buckets // 2 if both else buckets
    near = n // 2
    for r in range(-distance, distance + 1):
        dist, base = (abs(r), n if r > 0 else 0) if both else (max(-r, 0), 0)
        exact = dist if dist < near else near + math.log(dist / near) / math.log(distance / near) * (n - near)
        got = table[r + distance] - base
        want = min(math.floor(exact + 1e-9), n - 1)  # (a border is reached, never missed by a logarithm's last bit)
        assert got == want, r
    assert bucket_of(2, 3, table, 0, buckets)[0, 0] == table[distance]


def test_relative_buckets_refuses():
    import paper_2412_11007_amd as fs
    for bad in ((1, 10, False), (3, 10, True), (32, 8, True), (32, 2000, True), (130, 500, True), (7, 20, True)):
        with pytest.raises(ValueError):
            fs.fs_relative_buckets(*bad, device="cpu")
