"""The choices of hb_group_norm and hb_linear_i8 by size: what they promise whatever the sizes, and that the GPU tests take every form that they can choose."""
import random

import pytest

from featureforms import I8_FORMS, NORM_FORMS, ROWS, Plans, linear_form, norm_form


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    return Plans(tmp_path_factory.mktemp("plans"))


def sizes(rng):
    return lambda most: max(1, int(most ** rng.random()))


def norm_calls(seed, count, most=1 << 25):
    rng, calls = random.Random(seed), []
    size = sizes(rng)
    while len(calls) < count:
        G = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 5, 7, 64, size(300)])
        C = G * (size(4096) if rng.random() < 0.3 else size(128))
        N, P = size(1 << 16) if rng.random() < 0.3 else size(64), size(1 << 21)
        if N * P * C <= most:
            calls.append((N, P, C, G, rng.random() < 0.5, rng.random() < 0.6))
    return calls


def test_group_norm(plans):
    calls = norm_calls(1, 20000) + norm_calls(2, 5000, 1 << 45)
    calls += [(1, (1 << 30) - 1, 1, 1, 0, 1), (1, (1 << 30) - 1, 4096, 1, 1, 0), ((1 << 29) - 1, 1, 2, 2, 0, 1), (1, 1, 1 << 30, 1 << 29, 0, 1), (1, 1, 1, 1, 1, 0)]
    for (N, P, C, G, f32, dense), p in zip(calls, plans.group_norm(calls)):
        V, D, what = 4 if f32 else 8, C // G, (N, P, C, G, f32, dense, p)
        across = p["threads"] // (p["images"] * p["width"])
        assert p["threads"] in (64, 128, 256, 512, 1024) and across >= 1, what
        assert p["pixels"] in (1, 2, 4, 8) and (p["pixels"] == 1 or (dense and p["pixels"] * C % V == 0 and p["groups"] == G)), what
        assert (p["rows"] - 1) * p["pixels"] < P <= p["rows"] * p["pixels"], what
        assert 1 <= p["groups"] <= G and (p["blocks"] - 1) * p["groups"] < G <= p["blocks"] * p["groups"], what
        assert (p["width"] - 1) * V < p["pixels"] * p["groups"] * D <= p["width"] * V, what
        groups = p["images"] * p["groups"]
        assert p["log_lanes"] <= 6 and (p["threads"] >> p["log_lanes"]) >= 1 and (groups << p["log_lanes"]) < 2 * p["threads"] or p["log_lanes"] == 0, what
        E = 1 if D % V == 0 else 2 if D >= V else V
        if p["slab"]:
            assert (p["passes"] - 1) * across < p["rows"] <= p["passes"] * across and p["passes"] <= (14 if V == 8 and E > 1 else 16), what
            assert p["images"] == 1 or p["groups"] == G, what
            assert 4 * (2 * p["threads"] * E + 2 * groups) <= 160 * 1024, what
        else:
            for chunk, chunks in ((p["chunk"], p["chunks"]), (p["apply_chunk"], p["apply_chunks"])):
                assert (chunks - 1) * chunk < p["rows"] <= chunks * chunk and chunk % across == 0, what
                assert chunk < (1 << 30) + 4096 and (chunk << 3) < 1 << 34, what
            assert p["images"] == 1 and p["chunks"] <= 8 << (6 if p["join"] else p["log_lanes"]), what              # a lane joins eight
            assert N * G * (p["chunks"] + 1) * 8 <= p["workspace"] and p["workspace"] % 256 == 0, what
            assert 12 * p["threads"] * E <= 160 * 1024 and 8 * p["groups"] <= 65536, what


def test_every_form_of_group_norm_is_tested(plans):
    calls = norm_calls(3, 100000)
    reached = {norm_form(c, p): c for c, p in zip(calls, plans.group_norm(calls))}
    tested = {norm_form(c, p) for c, p in zip(NORM_FORMS, plans.group_norm(NORM_FORMS))}
    rare = {f: c for f, c in reached.items() if f not in tested}
    assert len(tested) >= 200 and len(reached) >= 150 and len(rare) <= 3, rare                  # combinations of two edges that a tenth of a million calls meet once


def test_linear_i8(plans):
    rng = random.Random(4)
    size = sizes(rng)
    calls = [(size(1 << 21), size(1 << 15), size(131071), rng.choice(ROWS)) for _ in range(5000)] + [(1, 1, 1, "odd"), ((1 << 31) - 256, 1, 1, "even"), (1, (1 << 31) - 1, 1, "odd"), (1, 1, 131071, "odd"),
                                                                                                    (1 << 30, 1 << 20, 64, "copied")]
    for (M, N, K, rows), (kernel, parts, per, need) in zip(calls, plans.linear_i8(calls)):
        steps = (K + 127) // 128
        assert 0 <= kernel <= 6 and parts >= 1 and (parts - 1) * per < steps <= parts * per, (M, N, K)            # no part is empty, none is missing
        assert kernel >= 3 or M <= (16, 32, 64)[kernel]
        assert kernel != 6 or (rows == "copied" and parts == 1)
        assert (parts == 1 or parts * M * N * 4 <= need <= 1 << 28) and need % 256 == 0, (M, N, K, parts, need)


def test_every_form_of_linear_i8_is_tested(plans):
    rng = random.Random(1)
    size, calls = sizes(rng), []
    while len(calls) < 100000:
        M, N, K, rows = size(1 << 20), size(1 << 14), size(1 << 15), rng.choice(ROWS)
        if M * max(N, K) <= 1 << 27:
            calls.append((M, N, (K + 15) // 16 * 16 if rows == "copied" else K, rows))
    reached = {linear_form(c, p) for c, p in zip(calls, plans.linear_i8(calls))}
    tested = {linear_form(c, p) for c, p in zip(I8_FORMS, plans.linear_i8(I8_FORMS))}
    assert len(reached) >= 20 and reached <= tested, sorted(reached - tested)
    assert all(rows != "copied" or K % 16 == 0 for _, _, K, rows in I8_FORMS)
