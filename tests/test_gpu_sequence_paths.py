"""The operators on sequences on the paths that large batches take, on batches small enough for the reference: convolution runs of
several rows and sequences, scans of the longest sequences first, pieces of more than 64 sequences, rooms with a start and a length."""
import pytest
import torch

import sequence_reference as ref
from paper_1907_02129_amd import binding as icv
from test_gpu_sequence import Batch, conv_case, gen, scan_case

pytestmark = pytest.mark.gpu


def ragged(count, mean, seed):
    """Lengths that spread over a factor of about ten around their mean, with empty ones, single rows and equal ones."""
    n = (torch.exp(torch.randn(count, generator=gen(seed)) * 0.8 - 0.3) * mean).int().tolist()
    for i in range(0, count, 7):
        n[i] = 0
    for i in range(3, count, 11):
        n[i] = 1
    for i in range(5, count - 2, 9):
        n[i + 2] = n[i]
    return n


def rooms(lengths, spare, seed):
    """Rooms of different size one behind the other, with rows in front of the first and behind the last, and of each only the first
    `lengths` rows in use; a length outside the room counts as the nearer bound."""
    batch = Batch(lengths)
    free = torch.randint(0, spare + 1, (len(lengths),), generator=gen(seed)).tolist()
    at = [3]
    for n, f in zip(lengths, free):
        at.append(at[-1] + n + f)
    batch.start, batch.tokens = at, at[-1] + 5
    batch.length = [-4 if n == 0 and i % 2 else (n + 9 if f == 0 else n) for i, (n, f) in enumerate(zip(lengths, free))]
    batch.rows = ref.spans(batch.count, batch.tokens, batch.start, batch.length)
    assert [n for _, n in batch.rows] == list(lengths)
    return batch


LONG = [5, 0, 1, 70, 2, 0, 33, 64, 31, 32, 1, 100, 3, 0, 0, 9]
PATHS = {
    "packed_in_place": Batch(LONG, "packed", tail=41),
    "packed_to_other_slots": Batch(LONG, "packed", tail=1, source=[i if i % 3 else -1 for i in range(16)], target=[31 - i if i % 5 else -1 for i in range(16)],
                                   slots=32),
    "one_prefix": Batch(LONG, "packed", source=[0] * 16, target=list(range(1, 17)), slots=17),
    "padded": Batch([17, 0, 64, 1, 3, 66, 2], "padded", tail=2),
    "short_ones": Batch([(i * 7) % 5 for i in range(90)], "packed", tail=3),
    "equal": Batch([40] * 5, "packed"),
    "rooms": rooms(LONG, 6, 1),
    "one_long": Batch([333]),
}


@pytest.mark.parametrize("run", [1, 2, 4, 8, 16, 32])
@pytest.mark.parametrize("name", list(PATHS))
def test_convolution_runs(run, name, monkeypatch):
    """Every number of rows a run may have (test hook): several sequences in a run, borders, empty sequences and rows of none inside one,
    rows that the old state reaches past a run's end, states from runs of several rows."""
    make = icv.make_causal_conv_params

    def hooked(*args, **kw):
        p = make(*args, **kw)
        p.silu |= run << 8
        return p

    monkeypatch.setattr(icv, "make_causal_conv_params", hooked)
    for dtype in ("bf16", "f32"):
        for channels, taps, silu, pad in ((72, 4, True, 0), (23, 2, False, 1), (3, 8, True, 2), (1, 3, False, 0), (21, 8, True, 0)):
            conv_case(PATHS[name], channels, taps, dtype, silu, taps != 3, True, pad, run + taps)
            if name in ("packed_in_place", "rooms"):
                conv_case(PATHS[name], channels, taps, dtype, silu, taps == 3, False, pad, run)


@pytest.mark.parametrize("dtype,channels", [("bf16", 8200), ("f32", 4103)])
def test_convolution_of_a_large_ragged_batch(dtype, channels):
    """Enough rows and channels for runs of 32 rows by the library's own choice."""
    lengths = ragged(24, 90, 2)
    lengths[-1] += 2100 - sum(lengths)
    assert lengths[-1] > 0
    conv_case(Batch(lengths, "packed", tail=37, source=[i if i % 2 else -1 for i in range(24)], target=[24 + i for i in range(24)], slots=48),
              channels, 4, dtype, True, True, True, 0, 3)
    conv_case(rooms(lengths, 9, 4), channels, 3, dtype, False, True, True, 1, 4)


@pytest.mark.parametrize("name", list(PATHS) + ["start_and_length_of_single_rows"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scan_rooms_and_prefixes(name, dtype):
    batch = PATHS[name] if name in PATHS else rooms([1, 0, 1, 1, 0, 1], 2, 5)
    for states, hook in ((16, 0), (13, 1), (16, 3), (16, 1 | 1 << 2), (13, 2 | 1 << 2), (3, 1 | 2 << 2)):
        scan_case(batch, 22, states, 2, dtype, True, True, True, 1, states, scale=0.1, hook=hook)


@pytest.mark.parametrize("layout", ["packed", "padded", "rooms"])
@pytest.mark.parametrize("count,per_lane", [(20, 3), (41, 2), (63, 3), (64, 1), (64, 3)])
def test_scan_longest_sequences_first(layout, count, per_lane):
    """More than 256 workgroups and 32 rows a sequence on the average: sequences in the order of their lengths, equal and empty ones
    among them.  `per_lane`: the hook for four, two or one of 16 states a lane, so 64, 32 or 16 channels a workgroup."""
    width = {1: 64, 2: 32, 3: 16}[per_lane]
    lengths = ragged(count, 38, count)
    if layout == "padded":
        batch = Batch(lengths, "padded", tail=1)
    else:
        lengths[-1] += max(0, 33 * count - sum(lengths))
        batch = Batch(lengths, "packed", tail=2) if layout == "packed" else rooms(lengths, 3, count)
    channels = width * (256 // count + 1)
    assert batch.tokens // count >= 32 and channels // width * count > 256 and len(set(lengths)) < count
    assert scan_case(batch, channels, 16, 1, "bf16", True, True, True, 0, count, scale=0.1, hook=per_lane) == 0


@pytest.mark.parametrize("count", [65, 128, 129, 200])
@pytest.mark.parametrize("layout", ["packed", "padded", "rooms"])
def test_scan_pieces_of_many_sequences(count, layout):
    """Pieces of 64 rows of more than 64 sequences, of no piece, one and several each."""
    lengths = [n if n < 400 else 400 for n in ragged(count, 50, count + 1)]
    if layout == "padded":
        lengths = [min(n, 140) for n in lengths]
    assert max(lengths) > 128 and 0 in lengths and 1 in lengths
    batch = {"packed": lambda: Batch(lengths, "packed", tail=9, source=[(i * 3) % count for i in range(count)], target=[count + i for i in range(count)],
                                     slots=2 * count),
             "padded": lambda: Batch(lengths, "padded", tail=1), "rooms": lambda: rooms(lengths, 4, count)}[layout]()
    for code, dtype in ((1, "bf16"), (3, "f32")):
        assert scan_case(batch, 18, 16, 1, dtype, True, True, True, 0, count, scale=0.02, hook=code | 1 << 2) > 0
