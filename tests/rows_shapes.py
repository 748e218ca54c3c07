"""Calls whose plan takes a form of the kernel that smaller ones do not reach: 256 query rows to a workgroup, over more tiles of 64 keys than
its ring holds and more blocks than one window of places, in one range and in several; more sequences than a launch has, with several ranges in
each launch.  tests/test_rows_plan.py checks that they are planned so, tests/test_gpu_rows_wide.py that they are right."""

TILE = 64
WINDOW = 1024        # keys whose places are looked up at once
RING = 4             # tiles

# (query heads, kv-heads, tokens, states, ranges that are expected): `several` or one; keys of a range, at least
WIDE_CROSS = [
    (32, 8, 1025, 300, False, RING * TILE + 1),
    (64, 64, 129, 5000, True, WINDOW + 1),
    (64, 64, 1000, 1200, False, WINDOW + 1),
]
# the same in sequences of unlike lengths, some of 32 rows and fewer: (query heads, kv-heads, tokens of each, states of each)
WIDE_RAGGED = (64, 64, [256, 0, 256, 5, 1], [2500, 40, 1100, 0, 2000])
# (query heads, kv-heads, sequences, slots of the prefix, keys of a range, at least)
WIDE_SHARED = [
    (64, 16, 33, 5000, RING * TILE + 1),
    (256, 32, 17, 2500, RING * TILE + 1),
    (256, 64, 33, 5000, WINDOW + 1),
]


def own_slots(n):
    return [(i * 7) % 40 for i in range(n)]


def many_sequences(n=70):
    """Tokens and states: the first two launches of 32 have sequences of several ranges, of 32 rows of a kv-head with two query heads and of more."""
    q_len = [20 if i % 18 == 0 else 3 if i % 18 == 9 else (i * 5) % 9 for i in range(n)]
    return q_len, [6000 + 13 * i if i % 9 == 0 else (i * 37) % 150 for i in range(n)]


# prefixes, sequences of each, own slots: more of all than a launch has, prefixes of very unlike lengths, in another order than their sequences' own
def many_prefixes(n=21):
    sharing = [(i * 5) % 7 for i in range(n)]
    sharing[3], sharing[17] = 40, 25
    prefix = [(i * 411) % 900 for i in range(n)]
    prefix[3], prefix[11], prefix[18] = 9000, 5000, 7000
    own = [(i * 13) % 70 for i in range(sum(sharing))]
    own[5], own[70], own[-1] = 3000, 2500, 4000
    return prefix, sharing, own
