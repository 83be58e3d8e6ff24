"""The choice of the 8-bit products' kernel: that the sizes which the tests on a GPU name for each kernel go there, and what holds for all sizes."""
import random

import pytest

from tests import eight_plan as P


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return P.load(tmp_path_factory.mktemp("plan"))


EVERY = [dict(dtype=d, eight=e, vectors=v, masked=m) for d in ("bf16", "f32") for e in (False, True) for v in (False, True) for m in (False, True)]


def test_the_lists_reach_what_they_name(lib):
    for how in EVERY:
        for (rows, ranks), size in P.FEW.items():
            assert P.plan(lib, *size, **how) == ("few", rows, ranks), (size, how)
        for size in P.ONE:
            assert P.plan(lib, *size, **how) == ("one",), (size, how)
        for size in P.PAIR:
            assert P.plan(lib, *size, **how) == ("pair",), (size, how)
        assert P.plan(lib, *P.MASKED_TO_PAIR, **how) == (("pair",) if how["masked"] else ("one",))
        assert P.plan(lib, *P.MASKED_TO_ONE, **how) == (("one",) if how["masked"] else ("pair",))


def test_few_rows_do_not_depend_on_the_mask_and_sums_are_never_too_long(lib):
    rng = random.Random(1)
    for _ in range(3000):
        m, n, k = (int(2 ** rng.uniform(0, top)) for top in (14.5, 14.5, 18))
        how = dict(dtype=rng.choice(["bf16", "f32"]), eight=rng.random() < 0.4, vectors=rng.random() < 0.7)
        plain, masked = P.plan(lib, m, n, k, **how), P.plan(lib, m, n, k, masked=True, **how)
        assert (plain[0] == "few") == (masked[0] == "few") and (plain[0] != "few" or plain == masked)
        exact = how["dtype"] == "f32" and not how["eight"]
        blocks = -(-k // 128)
        share = -(-blocks // plain[2]) if plain[0] == "few" else blocks
        assert share <= (max(64, blocks // 8 + 1) if exact else 256)
        if plain[0] == "few":
            assert plain[1] in (16, 32, 64, 128) and plain[2] in (1, 2, 4, 8)


def test_the_largest_sizes_are_planned_in_64_bits(lib):
    most = (1 << 31) - (1 << 16)
    for size in ((most, 1, 1), (1, most, 1), (1, 1, 262144), (most, most, 262144)):
        for how in EVERY:
            assert P.plan(lib, *size, **how)[0] in ("few", "one", "pair")
