"""What the sequence operators' entry points launch for a call, on the CPU (tests/host_sequence_launches.cpp): the limits that a launch
has, and the kernels that the rules of linear attention choose."""
import re

import pytest

from paper_2501_08455_amd import binding
from test_host_sanitized import linked, run   # noqa: F401 (a fixture)

F32, BF16, F16 = binding.SIG_F32, binding.SIG_BF16, binding.SIG_F16
OK, LARGE = binding.SIG_OK, binding.SIG_ERR_TOO_LARGE


class Launch:
    def __init__(self, words):
        self.kernel, *sizes = words.split(",")
        self.grid, self.threads = tuple(int(n) for n in sizes[:3]), int(sizes[3])
        self.workgroups = self.grid[0] * self.grid[1] * self.grid[2]


@pytest.fixture(scope="module")
def launches(linked):   # noqa: F811
    """launches(calls): (status, most bytes asked for, launches) of each"""
    exe = linked("host_sequence_launches.cpp")

    def answers(calls):
        lines = run(exe, calls="".join(" ".join(str(word) for word in call) + "\n" for call in calls)).splitlines()
        assert len(lines) == len(calls)
        return [(int(line.split()[0]), int(line.split()[1]), [Launch(w) for w in line.split()[2:]]) for line in lines]

    return answers


def within_limits(launch):
    """A launch holds fewer than 2^32 threads along an axis, and up to 65,535 workgroups along the second and third."""
    return launch.grid[0] * launch.threads < 1 << 32 and launch.grid[1] < 1 << 16 and launch.grid[2] < 1 << 16


HUGE = [("rotary", 1 << 14, 1 << 14, 1, 2, 2, BF16), ("rotary", 1, (1 << 28) + 5, 1, 8, 4, BF16), ("rotary", (1 << 24) + 1, 1, 1, 4096, 4096, BF16),
        ("rotary", 1, (1 << 31) - 1, 1, 2, 0, BF16)]
HUGE += [(way, *shape, kind) for way in ("forward", "backward") for kind in (F32, BF16)
         for shape in (((1 << 24) + 3, 1, 1, 1, 1, 1), ((1 << 24) + 3, 40, 1, 1, 8, 8), (1 << 23, 5, 4, 2, 4, 100), ((1 << 31) - 1, 1, 1, 1, 2, 1),
                       (1 << 21, 3, 9, 3, 200, 1), (1, 70, (1 << 24) - 1, 1, 4, 4))]


def test_no_launch_is_larger_than_launches_are(launches):
    for call, (rc, _, got) in zip(HUGE, launches(HUGE)):
        assert rc == OK and got, call
        for launch in got:
            assert within_limits(launch), (call, launch.kernel, launch.grid, launch.threads)


def test_what_no_launch_can_hold_is_refused(launches):
    calls = [(way, 1, 70, 1 << 24, 1, 4, 4, F32) for way in ("forward", "backward")]
    calls += [(way, 1 << 20, 1 << 17, F32) for way in ("norm", "norm_backward")] + [("norm_backward", 0, 1 << 31, F32), ("rotary", 1 << 16, 1 << 15, 1, 2, 2, F32)]
    for call, (rc, _, got) in zip(calls, launches(calls)):
        assert rc == LARGE and not got, (call, rc)


def test_slices_of_a_batch_hold_all_of_it(launches):
    """Token by token a workgroup is a head's 64 columns: as many of them as there are, over all launches of a pass."""
    B, H, V = (1 << 23) + 7, 5, 130
    ((rc, _, got),) = launches([("forward", B, 1, H, H, 4, V, F32)])
    assert rc == OK and len(got) > 1
    assert sum(launch.workgroups for launch in got) == B * H * 3 and all("recurrent" in launch.kernel for launch in got)


def test_rows_of_any_number_are_normalised(launches):
    for rc, _, got in launches([("norm", 1 << 33, 2, BF16), ("norm_backward", 1 << 33, 2, BF16), ("norm", 1 << 15, 16385, F32)]):
        assert rc == OK and got and all(within_limits(launch) for launch in got)


def test_shared_heads_gradients_take_no_more_than_8_gib_of_scratch(launches):
    """... by slices of the batch, each with all launches of the gradient."""
    small, large, one = ("backward", 8, 4096, 16, 4, 128, 128, BF16), ("backward", 100, 65536, 16, 4, 128, 128, BF16), ("backward", 1, 1 << 20, 16, 4, 128, 128, BF16)
    (a, few, whole), (b, many, cut), (c, most, single) = launches([small, large, one])
    assert a == b == c == OK
    parts = 4 * 16 * 256
    assert 8 * 4096 * parts <= few < 8 * 4096 * parts + (1 << 28)
    # a batch element of the second takes 1 GiB: slices of eight
    assert 8 * 65536 * parts <= many < (8 << 30) + (1 << 28)
    assert sum("sig_attention_share" in launch.kernel for launch in cut) == 2 * 13 and sum("sig_attention_share" in launch.kernel for launch in whole) == 2
    # a single sequence cannot be taken apart
    assert (1 << 20) * parts <= most and sum("sig_attention_share" in launch.kernel for launch in single) == 2


class Chunks:
    """How a call's chunk launches are cut: tiles of 16 columns a wavefront (64 nv columns a workgroup) and segments along time."""

    def __init__(self, launched, passes=1):
        found = [(re.search(r"Li(\d+)ELi(\d+)ELi(\d+)ELb([01])E", launch.kernel), launch) for launch in launched if "attention_chunk" in launch.kernel]
        (sizes, launch), = [x for x in found if x[0].group(4) == "1"]      # the launch with output
        self.columns, self.segments, self.workgroups = 64 * int(sizes.group(3)), launch.grid[2] // passes, launch.workgroups
        assert len(found) == (2 if self.segments > 1 else 1)


# B, T, heads, K, V, type: whether a sequence is cut along time.  256 compute units
CUT = [
    # as many workgroups of 64 columns as units, or up to twice as many: bfloat16 states of 128 rows, long sequences, where three segments of 128 columns fit
    ((8, 4096, 16, 128, 128, BF16), 4), ((1, 8192, 100, 128, 128, BF16), 5), ((1, 4096, 140, 128, 128, BF16), 3), ((1, 4096, 200, 128, 128, BF16), 1),
    ((8, 2048, 16, 128, 128, BF16), 1), ((1, 4096, 200, 128, 64, BF16), 2), ((1, 4096, 256, 96, 64, BF16), 2), ((1, 4096, 300, 128, 64, BF16), 1),
    ((1, 8192, 256, 256, 64, BF16), 1), ((1, 8192, 128, 192, 128, BF16), 1),
    # small ones from 2,048 tokens on
    ((50, 2048, 4, 64, 64, BF16), 3), ((50, 1024, 4, 64, 64, BF16), 1),
    # float32 states of more than 96 rows
    ((50, 2048, 4, 128, 64, F32), 1), ((50, 2048, 4, 192, 64, F32), 1), ((50, 2048, 4, 256, 64, F32), 1),
]


def test_sequences_are_cut_where_that_was_measured_to_pay(launches):
    got = launches([("forward", B, T, H, H, K, V, kind) for (B, T, H, K, V, kind), _ in CUT])
    wrong = [(call, segments, Chunks(launched).segments) for (call, segments), (rc, _, launched) in zip(CUT, got) if rc != OK or Chunks(launched).segments != segments]
    assert not wrong, wrong


def test_float32_sequences_of_one_workgroup_a_unit_stay_whole(launches):
    """... where that is 64 columns each; more workgroups than units, or wider states, are cut."""
    shapes = [((200, 64, 64), 1), ((256, 64, 64), 1), ((256, 96, 64), 1), ((280, 64, 64), 2), ((100, 64, 128), 5), ((400, 64, 64), 1)]
    got = launches([("forward", 1, 4096, H, H, K, V, F32) for (H, K, V), _ in shapes])
    for (shape, segments), (rc, _, launched) in zip(shapes, got):
        assert rc == OK and Chunks(launched).segments == segments, (shape, Chunks(launched).segments)


def test_short_sequences_of_few_heads_keep_their_workgroups(launches):
    """64 columns a workgroup where time has too few pieces for 128 to fill the units: twice the workgroups for the units that idle."""
    shapes = [((4, 192, 8, BF16), 64, 1), ((1, 300, 8, F32), 64, 2), ((1, 1000, 24, BF16), 64, 4), ((1, 8000, 8, BF16), 64, 25), ((1, 65536, 8, BF16), 128, 64),
              ((1, 4096, 48, BF16), 128, 10), ((1, 16384, 8, F32), 128, 64)]
    got = launches([("forward", B, T, H, H, 128, 128, kind) for (B, T, H, kind), _, _ in shapes])
    for (shape, columns, segments), (rc, _, launched) in zip(shapes, got):
        cut = Chunks(launched)
        assert rc == OK and (cut.columns, cut.segments) == (columns, segments), (shape, cut.columns, cut.segments)
        assert cut.workgroups == shape[0] * shape[2] * 128 // columns * segments
