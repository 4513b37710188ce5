"""The sizes of the GPU test of every kind of tiles take the kinds that they claim, and no kind is left out."""
import pytest

from tests.tile_kinds import BIG_DEPTHS, BIG_LAST, SIZES, big_sizes, compile_rule


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return compile_rule(tmp_path_factory.mktemp("plan"))


@pytest.mark.parametrize("form,elem,result,kind,parts,E,N,K,R", SIZES)
def test_sizes_take_their_kind(plan, form, elem, result, kind, parts, E, N, K, R):
    tiles, n = plan(form, elem, result, E, N, K, R)
    assert (tiles, "one" if n == 1 else "several") == (kind, parts)


def test_every_kind_has_its_sizes():
    products = [("forward", "bf16", "bf16"), ("forward", "f32", "f32"), ("input_grad", "bf16", "bf16"), ("input_grad", "f32", "f32"),
                ("weight_grad", "bf16", "bf16"), ("weight_grad", "bf16", "f32"), ("weight_grad", "f32", "f32"), ("weight_grad", "f32", "bf16"),
                ("forward", "i8", "bf16"), ("forward", "i8", "f32")]
    want = set()
    for p in products:
        for kind in ("mid", "slim", "big", "few"):
            for parts in ("one", "several"):
                if kind == "big" and p[1] == "f32" or kind == "few" and p[0] == "weight_grad":
                    continue  # no kernel
                if kind == "slim" and (p[0] != "weight_grad" or parts == "several"):
                    continue
                want.add((*p, kind, parts))
    assert {s[:5] for s in SIZES} == want


def test_depths_of_the_largest_tiles(plan):
    for last in BIG_LAST:
        E, N, R = big_sizes(last)
        assert all(plan("forward", "bf16", "bf16", E, N, depth, R) == ("big", 1) for depth in BIG_DEPTHS)


def test_the_rule_takes_no_other_kind(plan):
    """Over sizes of every magnitude."""
    import random
    rng, seen = random.Random(1), {s[:5] for s in SIZES}
    for _ in range(3000):
        form, elem, result = rng.choice(SIZES)[:3]
        E, N, K, R = (int(2 ** rng.uniform(0, top)) for top in (7, 14, 14, 15))
        tiles, n = plan(form, elem, result, E, N, K, R)
        assert (form, elem, result, tiles, "one" if n == 1 else "several") in seen
