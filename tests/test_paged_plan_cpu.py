"""The dealing of whole query tiles to workgroups (dkv_paged_query_attn's plan)
on the host: whether a call takes that form is a function of its lengths.

The plan sorts the units by falling length into 1,024 buckets, where those of
one bucket stand in the order of arrival, deals them P at a time and takes the
form when the longest share is near enough to the mean.  `deal` follows it with
the order within the buckets as an argument, and with each unit counted by its
own length or by its bucket's longest."""

import numpy as np
import pytest

ROWS, TILE, OVERHEAD, SLICES, BUCKETS = 256, 64, 2, 256, 1024


def unit_costs(held, new, Hkv, G):
    """Costs of the units, sequence by sequence and head by head, of a cache whose pages are all there."""
    out = []
    for h, n in zip(held, new):
        mine = []
        for qt in range(-(-n * G // ROWS)):
            sees = h + (min((qt + 1) * ROWS, n * G) - 1) // G + 1
            left = n * G - qt * ROWS
            cost = 2 if left <= 64 else (3 if left <= ROWS // 2 else 4)
            mine.append((-(-sees // TILE) + OVERHEAD) * cost)
        out += mine * Hkv
    return np.array(out, dtype=np.int64)


def deal(cost, own_length, rng=None, P=SLICES):
    """Whether the units are taken whole; rng shuffles the units of each bucket."""
    units, total, longest = len(cost), int(cost.sum()), int(cost.max())
    if units <= P or units > 4096 or longest > total // P or units > 32 * P or total < units * 10 * 4:
        return False
    scale = np.float32(BUCKETS - 1) / np.float32(longest)
    bucket = np.minimum(((longest - cost).astype(np.float32) * scale).astype(np.int64), BUCKETS - 1)
    arrival = np.arange(units) if rng is None else rng.permutation(units)
    order = arrival[np.argsort(bucket[arrival], kind="stable")]
    most = np.zeros(BUCKETS, dtype=np.int64)
    np.maximum.at(most, bucket, cost)
    size = cost if own_length else most[bucket]
    load = np.zeros(P, dtype=np.int64)
    for r in range(-(-units // P)):
        by_load = np.argsort(load, kind="stable") if r > 1 else np.arange(P)[::-1 if r else 1]
        mine = order[r * P:(r + 1) * P]
        load[by_load[:len(mine)]] += size[mine]
    return bool(load.max() <= total // P + 10 * 4)


# Query heads 32 on 8.  In the first two the longest share is just above the limit or at it by the order: 12,512 or
# 12,516 against 12,513, and 8,468 or 8,472 against 8,471.
BATCHES = [([65727, 65766, 64237], [1904, 2405, 1763]), ([66106, 66993], [2148, 1877]), ([0, 0], [4096, 4096]),
           ([0] * 8, [1500] * 8), ([20000] * 6, [1024] * 6), ([40000, 41000, 300, 9000], [2900] * 4)]


@pytest.mark.parametrize("batch", BATCHES[:2])
def test_counted_by_their_own_lengths_the_order_decides(batch):
    cost = unit_costs(*batch, 8, 4)
    rng = np.random.default_rng(0)
    assert len({deal(cost, True, rng) for _ in range(200)}) == 2


@pytest.mark.parametrize("batch", BATCHES)
def test_counted_by_their_bucket_it_does_not(batch):
    cost = unit_costs(*batch, 8, 4)
    rng = np.random.default_rng(1)
    assert len({deal(cost, False, rng) for _ in range(50)}) == 1


def test_random_batches_do_not_depend_on_the_order():
    rng = np.random.default_rng(2)
    for _ in range(40):
        B = int(rng.integers(1, 9))
        cost = unit_costs(rng.integers(0, 70000, size=B).tolist(), rng.integers(200, 4097, size=B).tolist(), 8, 4)
        assert len({deal(cost, False, rng) for _ in range(4)}) == 1


@pytest.mark.parametrize("hint", [0, -1])
@pytest.mark.parametrize("B,Hkv", [(2, 8), (1, 16), (3, 8), (16, 8), (256, 1), (32, 8)])
@pytest.mark.parametrize("new", [5, 8, 16])
def test_an_unknown_hint_is_a_long_cache(B, Hkv, new, hint):
    """33 to 128 query rows per segment and no hint: up to 16 segments the kernels for short blocks, as with long ones
    that they take, and beyond the query tiles, as with the longest; each has a workspace of its own size."""
    import paper_2609_32663_amd as d
    size = lambda h: d.dkv_paged_query_workspace_bytes(B, 8 * Hkv, Hkv, 128, B * new, new, h)  # noqa: E731
    assert size(hint) == size((1 << 18) - 1 if B * Hkv <= 16 else 1 << 40)
    assert size((1 << 18) - 1) != size(1 << 40) or B * Hkv > 16


def test_a_longest_chunk_beyond_int32_is_all_tokens():
    """The binding passes 32 bits; a bound above the number of tokens says nothing more than that number."""
    import paper_2609_32663_amd as d
    size = lambda most: d.dkv_paged_query_workspace_bytes(3, 32, 8, 128, 700, most, 0)  # noqa: E731
    assert size(700) > 0 and size(1 << 32) == size(700) and size((1 << 32) + 5) == size(700) != size(5)
