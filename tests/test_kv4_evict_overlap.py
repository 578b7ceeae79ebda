"""Where an eviction may write what it leaves of lengths, positions and weights (no GPU is touched: every call ends before a launch): over the array that it reads the same of,
or over nothing that it reads or writes else."""
import itertools

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_attention_arguments import P, _Kept, cache, ref, sequences

# sequences(): 3 of up to 4 pages of 32 places, 2 heads; arrays of (3, 2, 128) with strides 256 and 128: 768 elements, lengths 12 bytes, the table 48
BYTES = 4 * 768
LENGTHS, POSITIONS, WEIGHTS, TABLE = P << 3, P << 4, P << 5, P << 6
FREE = dict(lengths=P << 7, positions=P << 8, positions_sequence=256, positions_head=128, weights=P << 9, weights_sequence=256, weights_head=128)


def evict(to, **more):
    on = sequences(**dict(dict(lengths=LENGTHS, positions=POSITIONS, weights=WEIGHTS, table=TABLE), **more))
    kept = _Kept(*(dict(FREE, **to)[name] for name, _ in _Kept._fields_))
    return oz.lib().oz2_kv4_evict(ref(cache()), ref(on), 4, 0, ref(kept), None)


@pytest.fixture(autouse=True)
def no_workspace():
    oz.set_workspace(None, 0)


def test_apart_or_the_same():
    assert evict({}) == 1  # (no workspace: all else is well)
    same = dict(lengths=LENGTHS, positions=POSITIONS, weights=WEIGHTS)
    for n in (1, 2, 3):
        for names in itertools.combinations(same, n):
            assert evict({k: same[k] for k in names}) == 1
    for name, size, on in (("lengths", 12, LENGTHS), ("positions", BYTES, POSITIONS), ("weights", BYTES, WEIGHTS)):
        for at in (on - size, on + size):
            assert evict({name: at}) == 1


SIZES = dict(lengths=12, positions=BYTES, weights=BYTES)
INPUTS = dict(lengths=(LENGTHS, 12), positions=(POSITIONS, BYTES), weights=(WEIGHTS, BYTES), table=(TABLE, 48))


@pytest.mark.parametrize("to", SIZES)
@pytest.mark.parametrize("on", INPUTS)
def test_over_a_part_of_what_is_read(on, to):
    at, size = INPUTS[on]
    for by in (0, 4, size - 4, 4 - SIZES[to], (size - SIZES[to]) // 8 * 4):
        if on != to or by:
            assert evict({to: at + by}) == -5, by
    for by in (size, -SIZES[to]):
        assert evict({to: at + by}) == 1


def test_over_each_other():
    for a, b in itertools.permutations(SIZES, 2):
        for by in (0, 4, SIZES[a] - 4, 4 - SIZES[b]):
            assert evict({b: FREE[a] + by}) == -5
        assert evict({b: FREE[a] + SIZES[a]}) == 1


def test_other_strides_over_the_same_array():
    assert evict(dict(positions=POSITIONS, positions_sequence=512)) == -5 and evict(dict(weights=WEIGHTS, weights_head=130, weights_sequence=512)) == -5


def test_parts_of_one_packed_array():
    """(3, 2, 4, 128): old and new positions and weights, head by head; (3, 4, 2, 128): sequence by sequence; (4, 3, 2, 128): all of each behind all of another"""
    for sequence, head, step in ((1024, 512, 512), (1024, 128, 1024), (256, 128, BYTES)):
        at = [P << 10 | i * step for i in range(4)]
        strides = dict(positions_sequence=sequence, positions_head=head, weights_sequence=sequence, weights_head=head)
        assert evict(dict(positions=at[2], weights=at[3], **strides), positions=at[0], weights=at[1], **strides) == 1
        for by in (4, -4):
            assert evict(dict(positions=at[2] + by, weights=at[3], **strides), positions=at[0], weights=at[1], **strides) == -5


def test_what_is_refused_shares_bytes_and_what_is_not_does_not():
    """small arrays at random places, against the bytes that they have"""
    rng = np.random.default_rng(1)
    cover = lambda at, s, h: {at + 4 * (i * s + j * h + k) for i in range(3) for j in range(2) for k in range(128)}
    for _ in range(300):
        head = int(rng.choice([128, 130, 256, 384, 512]))
        sequence = int(rng.choice([2 * head, 2 * head + 6, 4 * head, 1024 + 2 * head]))
        if rng.random() < 0.3:
            head, sequence = sequence + 256, head
            if head < 3 * sequence:
                continue
        strides = dict(positions_sequence=sequence, positions_head=head)
        at = POSITIONS + 4 * int(rng.integers(-1500, 1500))
        shared = cover(POSITIONS, sequence, head) & cover(at, sequence, head)
        rc = evict(dict(positions=at, **strides), **strides)
        assert rc in ((1,) if at == POSITIONS else (-5,) if shared else (1, -5))


def test_strides_of_a_single_sequence_and_of_a_huge_table_say_nothing():
    on = dict(sequences=1, positions_sequence=7, weights_sequence=0)
    assert evict(dict(positions=POSITIONS, positions_sequence=1 << 40, weights=WEIGHTS, weights_sequence=5), **on) == 1
    assert evict({}, table=1 << 52, ld_table=2 ** 62) == 1
