"""What chunkkv_cross_attention and chunkkv_shared_decode_attention launch, on the host: every key of a segment in one range, every partial row at a
place of its own in the workspace and joined from where it was written, the forms of the kernel that the GPU tests are there for."""
import json
import os
import random
import subprocess

import pytest

from paper_2502_00299_amd import build
from tests import rows_shapes as shapes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16 = 0, 1, 2
TYPES = [(dt, d) for dt in (F32, BF16, F16) for d in (64, 128)]


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(calls) -> what each launches."""
    out = tmp_path_factory.mktemp("plan")
    exe, obj = str(out / "rows_plan"), str(out / "rows_plan.o")
    kept = [os.path.join(build.OBJ, s.replace(".hip", ".o")) for s in build.SOURCES if not s.startswith("rows_")]
    if not all(map(os.path.exists, kept)):
        build.build(verbose=False)
    subprocess.run([build.HIPCC, "-x", "hip", *build.FLAGS, "--cuda-host-only", "-O1", "-c", os.path.join(ROOT, "tests", "rows_plan_main.cpp"), "-o", obj], check=True, capture_output=True)
    subprocess.run([build.HIPCC, "-o", exe, obj, *kept], check=True, capture_output=True)

    def call(calls):
        text = "".join(" ".join([c[0], *map(str, c[1:5]), *(str(n) for part in c[5:] for n in ([part] if isinstance(part, int) else part))]) + "\n" for c in calls)
        answers = [json.loads(x) for x in subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=120).stdout.splitlines()]
        assert len(answers) == len(calls)
        return answers
    return call


def cross(dt, hq, hkv, d, q_len, seqlen):
    return "cross", dt, hq, hkv, d, len(q_len), q_len, seqlen


def shared(dt, hq, hkv, d, prefix, sharing, own):
    return "shared", dt, hq, hkv, d, len(prefix), len(own), sharing, prefix, own


def align(x):
    return (x + 255) // 256 * 256


def partial_bytes(rows, d):
    return align(rows * 16) + align(rows * d * 4)


def check_launch(launch, dt, hkv, d):
    """Workgroups of a launch, its segments' ranges and tiles; -> (first partial row, rows) of each segment."""
    at, spans = 0, []
    pairs = 1 if launch["tile"] == 32 or (dt == F32 and d == 128) else 2
    for first, rows, most, _, splits, tiles, part, keys in launch["segments"]:
        assert first == at
        if rows == 0:
            assert splits == 0
        elif rows <= 32:
            at += -(-splits * hkv // pairs)
            assert tiles == 1
        else:
            at += splits * hkv * tiles
            assert launch["tile"] in (128, 256) and (tiles - 1) * launch["tile"] < rows <= tiles * launch["tile"]
        if rows:
            assert splits >= 1 and keys % 64 == 0 and keys * splits >= most and (splits == 1 or keys * (splits - 1) < most)
        spans.append((part, splits * hkv * rows if part >= 0 else 0))
    assert launch["blocks"] == at
    return spans


def apart(spans, rows):
    """Partial rows of different segments do not meet, and lie in a workspace of so many."""
    end = 0
    for part, n in sorted(x for x in spans if x[1] > 0):
        assert part >= end
        end = part + n
    assert end <= rows


def check_cross(answer, dt, hq, hkv, d, q_len, seqlen):
    g, launches, at = hq // hkv, answer["launches"], 0
    room = max(n for n in range(answer["bytes"] // (16 + 4 * d) + 1, -1, -1) if partial_bytes(n, d) <= answer["bytes"])
    tokens = [sum(q_len[:b]) for b in range(len(q_len))]
    while launches:
        rows, launches = launches[0], launches[1:]
        assert rows["kind"] == "rows" and rows["seq0"] % 32 == 0 and rows["seq0"] >= at
        at = rows["seq0"]
        apart(check_launch(rows, dt, hkv, d), room)
        joined, before = [], 0
        for i, (_, r, most, row0, splits, _, part, _) in enumerate(rows["segments"]):
            b = at + i
            assert (r, most) == (q_len[b] * g, seqlen[b]) and row0 == tokens[b] and (part >= 0) == (splits > 1)
            if part >= 0:
                joined.append([before, part, splits, r, tokens[b], 0, 0, 0, 0, tokens[b] * hq * d * (4 if dt == F32 else 2)])
                before += q_len[b]
        if joined:
            assert launches[0]["kind"] == "join" and launches[0]["segments"] == joined and launches[0]["tokens"] == before
            launches = launches[1:]
        else:
            assert not launches or launches[0]["kind"] == "rows"


def check_shared(answer, dt, hq, hkv, d, prefix, sharing, own):
    g, P = hq // hkv, len(prefix)
    room = max(n for n in range(answer["bytes"] // (16 + 4 * d) + 1, -1, -1) if partial_bytes(n, d) <= answer["bytes"])
    spans, of_prefix, of_own = [], {}, {}
    joins = [x for x in answer["launches"] if x["kind"] == "join"]
    for launch in answer["launches"]:
        if launch["kind"] == "join":
            continue
        spans += check_launch(launch, dt, hkv, d)
        for i, (_, r, most, row0, splits, _, part, _) in enumerate(launch["segments"]):
            if i < launch["prefixes"]:
                p = launch["prefix0"] + i
                assert r == (sharing[p] * g if prefix[p] else 0) and most == prefix[p] and row0 == sum(sharing[:p]) and p not in of_prefix
                of_prefix[p] = (part, splits, r)
            else:
                b = launch["seq0"] + i - launch["prefixes"]
                assert r == (g if own[b] else 0) and most == own[b] and row0 == b and b not in of_own
                of_own[b] = (part, splits, r)
    apart(spans, room)
    assert all(p in of_prefix for p in range(P) if prefix[p] and sharing[p]) and all(b in of_own for b in range(len(own)) if own[b])
    at = 0
    whose = [(p, i) for p in range(P) for i in range(sharing[p])]
    for join in joins:
        assert join["tokens"] == len(join["segments"])
        for n, (first, part, splits, rows, token, prefix_part, prefix_splits, prefix_rows, row0, out) in enumerate(join["segments"]):
            b, (p, i) = at + n, whose[at + n]
            assert first == n and token == b and out == b * hq * d * (4 if dt == F32 else 2)
            if own[b]:
                assert (part, splits, rows) == of_own[b]
            else:
                assert splits == 0
            if prefix[p]:
                assert (prefix_part, prefix_splits, prefix_rows) == of_prefix[p] and row0 == i * g
            else:
                assert prefix_splits == 0
        at += len(join["segments"])
    assert at == len(own)


def drawn(rng):
    hkv, g, d, dt = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 3, 4, 8, 33]), rng.choice([64, 128]), rng.choice([F32, BF16, F16])
    length = lambda top: rng.choice([0, 1, 64, 65]) if rng.random() < 0.2 else int(10 ** rng.uniform(0, top))
    return dt, hkv * g, hkv, d, length


def test_drawn_cross_calls(ask):
    rng = random.Random(1)
    calls = []
    for _ in range(600):
        dt, hq, hkv, d, length = drawn(rng)
        n, top = rng.choice([1, 2, 5, 31, 32, 33, 64, 65, 100]), rng.uniform(0.5, 3)
        calls.append((dt, hq, hkv, d, [length(top) for _ in range(n)], [length(4.5) for _ in range(n)]))
    for c, a in zip(calls, ask([cross(*c) for c in calls])):
        assert a["rc"] == 0
        check_cross(a, *c)


def test_drawn_shared_calls(ask):
    rng = random.Random(2)
    calls = []
    for _ in range(600):
        dt, hq, hkv, d, length = drawn(rng)
        sharing = [rng.choice([0, 1, 1, 2, 5, 20, 70]) for _ in range(rng.choice([1, 2, 7, 8, 9, 17, 40]))]
        sharing[rng.randrange(len(sharing))] += 1
        calls.append((dt, hq, hkv, d, [length(4.5) for _ in sharing], sharing, [length(3.5) for _ in range(sum(sharing))]))
    for c, a in zip(calls, ask([shared(*c) for c in calls])):
        assert a["rc"] == 0
        check_shared(a, *c)


@pytest.mark.parametrize("dt,d", TYPES)
def test_shapes_of_256_rows(ask, dt, d):
    """The shapes of tests/test_gpu_rows_wide.py are planned as that says."""
    for (hq, hkv, n, states, several, keys), a in zip(shapes.WIDE_CROSS, ask([cross(dt, hq, hkv, d, [n], [m]) for hq, hkv, n, m, _, _ in shapes.WIDE_CROSS])):
        launch = a["launches"][0]
        (_, rows, _, _, splits, _, _, each), = launch["segments"]
        assert launch["tile"] == 256 and (splits > 1) == several and min(each, states) >= keys, (hq, n, states)
    hq, hkv, n, m, _, _ = shapes.WIDE_CROSS[0]
    assert ask([cross(dt, hq, hkv, d, [n] * 5, [m] * 5)])[0]["launches"][0]["tile"] == 256
    hq, hkv, q_len, states = shapes.WIDE_RAGGED
    assert ask([cross(dt, hq, hkv, d, q_len, states)])[0]["launches"][0]["tile"] == 256
    for (hq, hkv, n, slots, keys), a in zip(shapes.WIDE_SHARED, ask([shared(dt, hq, hkv, d, [m], [n], shapes.own_slots(n)) for hq, hkv, n, m, _ in shapes.WIDE_SHARED])):
        assert a["launches"][0]["tile"] == 256 and a["launches"][0]["segments"][0][7] >= keys


@pytest.mark.parametrize("dt,d", TYPES)
def test_shapes_of_many_segments(ask, dt, d):
    q_len, states = shapes.many_sequences()
    a, = ask([cross(dt, 4, 2, d, q_len, states)])
    check_cross(a, dt, 4, 2, d, q_len, states)
    rows = [x for x in a["launches"] if x["kind"] == "rows"]
    for launch in rows[:2]:   # a join behind each, of narrow segments and of wide ones
        cut = [x[1] for x in launch["segments"] if x[4] > 1]
        assert min(cut) <= 32 < max(cut)
    assert len(rows) == 3 and [x["kind"] for x in a["launches"]][:4] == ["rows", "join"] * 2 and a["bytes"] > 256
    prefix, sharing, own = shapes.many_prefixes()
    a, = ask([shared(dt, 8, 2, d, prefix, sharing, own)])
    check_shared(a, dt, 8, 2, d, prefix, sharing, own)
    assert [x["kind"] for x in a["launches"]].count("rows") >= 3


@pytest.mark.parametrize("dt,d", TYPES)
def test_every_launch_is_planned_for_all_of_the_card(ask, dt, d):
    """More segments than a launch has: the launches run one behind the other, so each of them is cut as a call of its segments alone."""
    calls = [(8, 4, [1] * 64, [16384] * 64), (1, 1, [1] * 128, [16384] * 128), (32, 8, [40] * 70, [9000] * 70), (32, 8, [1 + i % 3 for i in range(100)], [200 + 199 * i for i in range(100)])]
    for hq, hkv, q_len, states in calls:
        launches = [x for x in ask([cross(dt, hq, hkv, d, q_len, states)])[0]["launches"] if x["kind"] == "rows"]
        assert len(launches) == -(-len(q_len) // 32)
        for i, launch in enumerate(launches):
            part = slice(32 * i, 32 * i + 32)
            alone = ask([cross(dt, hq, hkv, d, q_len[part], states[part])])[0]["launches"][0]
            assert launch["tile"] == alone["tile"] and launch["blocks"] == alone["blocks"] and [x[4] for x in launch["segments"]] == [x[4] for x in alone["segments"]]
    # long prefixes, eight to a launch: a workgroup to every second CU at least, which an eighth of that was
    for sharing in ([16] * 64, [1] * 64):
        own = [16] * sum(sharing)
        a, = ask([shared(dt, 32, 8, d, [8192] * 64, sharing, own)])
        check_shared(a, dt, 32, 8, d, [8192] * 64, sharing, own)
        for launch in (x for x in a["launches"] if x["kind"] == "rows" and x["prefixes"]):
            assert sum(n[4] * 8 for n in launch["segments"][:8]) >= 128
