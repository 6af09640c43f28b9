"""The shapes of norm_forms reach every kernel of the RMS norm (no GPU needed)."""
import norm_forms


def test_every_form_is_reached_and_loops():
    shapes = [s + (d,) for s in norm_forms.MANY + norm_forms.FEW for d in ("f32", "bf16")]
    many, few = set(), set()
    for (n, c, p, d), (vec, form, blocks, parts) in zip(shapes, norm_forms.plans(shapes)):
        assert blocks > 0 and parts > 0
        key = (d, p > 1, vec, form)
        few.add(key)
        units, at_once = (n * -(-p // 32), blocks) if p > 1 else (n, 4 * blocks)
        if units > 2 * at_once:
            many.add(key)
        elif (n, c, p) in norm_forms.MANY:
            raise AssertionError((n, c, p, d, vec, form, blocks))
    want = {(d, True, v, f) for d, v, most in (("f32", 4, 4), ("f32", 1, 5), ("bf16", 8, 4), ("bf16", 4, 4), ("bf16", 1, 5))
            for f in (-1, *range(most))}
    assert want <= many, want - many
    rows = {(d, False, v, f) for d, v, most in (("f32", 4, 4), ("f32", 1, 3), ("bf16", 8, 3), ("bf16", 1, 3)) for f in range(most)}
    assert rows <= many, rows - many
    loops = {("f32", False, 4, -1), ("f32", False, 1, -1), ("bf16", False, 8, -1), ("bf16", False, 1, -1)}
    assert loops <= few, loops - few
    assert few == want | rows | loops
