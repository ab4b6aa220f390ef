"""The cache attention's rule of sharing out (host functions, no GPU)."""

import random

import kv_rules
import test_gpu_kv_shapes as shapes


def _random(rng):
    d = rng.choice([64, 128, 256])
    hkv = rng.choice([1, 2, 3, 8, 16])
    return d, rng.choice([1, 2, 5, 16, 64, 256]), rng.choice([1, 2, 5, 8, 9, 33, 100, 500, 4099]), hkv, \
        hkv * rng.choice([1, 2, 3, 4, 5, 7, 8]), rng.choice([1, 15, 100, 700, 3000, 16001, 65521, 1 << 30]), \
        rng.choice([0, 0, 1, 50, 1024, 1 << 30])


def test_shares_cover_rows_and_tokens():
    rng = random.Random(4)
    for _ in range(4000):
        d, n, R, hkv, hq, most, window = _random(rng)
        mt, wt, tiles, splits, chunk = kv_rules.attend_shape(d, n, R, hkv, hq, most, window)
        rows = R * hq // hkv
        per = 16 * mt * (4 // wt if wt < 8 else 1)
        assert (tiles - 1) * per < rows <= tiles * per
        assert 1 <= splits <= 128 and chunk > 0 and chunk % (32 * wt) == 0
        if not window:
            assert splits * chunk >= most and (splits - 1) * chunk < most


def test_every_instance_has_a_case():
    found = set()
    rng = random.Random(5)
    for _ in range(20000):
        d, n, R, hkv, hq, most, window = _random(rng)
        mt, wt, _, splits, _ = kv_rules.attend_shape(d, n, R, hkv, hq, most, window)
        found.add((d, mt, wt, kv_rules.join_kind(splits)))
    have = {(c[2],) + shapes.shape_of(c) for c in shapes.SHAPES}
    for c in shapes.SHAPES:
        assert shapes.shape_of(c) == c[7], c
    # the instances of the attention, and of the join
    assert {f[:3] for f in found} == {f[:3] for f in have}
    assert {(f[0], f[3]) for f in found} == {(f[0], f[3]) for f in have}
    assert len({f[:3] for f in have}) == 12
