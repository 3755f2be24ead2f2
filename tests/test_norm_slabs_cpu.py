"""The calls of normslabs.py are what they say: every form of hb_group_norm's kernel for groups in registers, and where the first vectors end."""
import random

import pytest

from featureforms import NORM_FORMS, Plans, norm_form
from normslabs import NORM_SLABS, first_pixels, slab_form


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    return Plans(tmp_path_factory.mktemp("slabs"))


def test_every_form_in_registers_is_tested(plans):
    calls = [c[:6] for c in NORM_SLABS]
    tested = set()
    for call, p in zip(NORM_SLABS, plans.group_norm(calls)):
        assert p["slab"] and first_pixels(call[:6], p) == call[6], call
        tested.add(slab_form(call[:6], p))
    # fp16 and fp32; a vector of one group, of two, of more, the last two with whole vectors or not and with one pixel in a row or more; vectors of a lane
    kinds = {(V, 1, True, False) for V in (4, 8)} | {(V, kind, whole, shared) for V in (4, 8) for kind in (2, V) for whole in (False, True) for shared in (False, True)}
    held = {(str(n), False) for n in (1, 2, 3, 4)} | {(n, large) for n in ("5", "between", "most") for large in (False, True)}
    assert tested == {k + h for k in kinds for h in held}


def test_no_other_form_is_reached(plans):
    rng, calls = random.Random(7), []
    size = lambda most: max(1, int(most ** rng.random()))
    while len(calls) < 100000:
        G = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 5, 7, 64, size(300)])
        C = G * (size(4096) if rng.random() < 0.3 else size(128))
        N, P = size(1 << 16) if rng.random() < 0.3 else size(64), size(1 << 21)
        if N * P * C <= 1 << 25:
            calls.append((N, P, C, G, int(rng.random() < 0.5), int(rng.random() < 0.6)))
    tested = {slab_form(c, p) for c, p in zip([c[:6] for c in NORM_SLABS], plans.group_norm([c[:6] for c in NORM_SLABS]))}
    reached = {slab_form(c, p) for c, p in zip(calls, plans.group_norm(calls)) if p["slab"]}
    assert len(reached) > 150 and reached <= tested, sorted(reached - tested)


def test_first_vectors_are_a_16th_of_all(plans):
    """What bounds the squares about their mean."""
    for call in NORM_SLABS:
        assert 16 * call[6] >= call[1], call


def test_no_form_of_any_kernel_is_left_over(plans):
    """Those that stream among them, whose calls are featureforms.NORM_FORMS."""
    rng, calls = random.Random(8), []
    size = lambda most: max(1, int(most ** rng.random()))
    while len(calls) < 100000:
        G = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 5, 7, 64, size(300)])
        C = G * (size(4096) if rng.random() < 0.3 else size(128))
        N, P = size(1 << 16) if rng.random() < 0.3 else size(64), size(1 << 21)
        if N * P * C <= 1 << 25:
            calls.append((N, P, C, G, int(rng.random() < 0.5), int(rng.random() < 0.6)))
    listed = NORM_FORMS + [c[:6] for c in NORM_SLABS]
    tested = {norm_form(c, p) for c, p in zip(listed, plans.group_norm(listed))}
    reached = {norm_form(c, p): c for c, p in zip(calls, plans.group_norm(calls))}
    assert not {f: c for f, c in reached.items() if f not in tested}
