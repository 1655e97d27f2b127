"""What window attention's and the paged cache's entry points launch for a call, on the CPU (tests/host_window_launches.cpp): the limits that a launch has,
and the cuts that their rules choose."""
import re

import pytest

from paper_2501_08455_amd import binding
from test_host_sanitized import linked, run   # noqa: F401 (a fixture)
from test_host_sequence_launches import Launch, within_limits

F32, BF16, F16, E4M3 = binding.SIG_F32, binding.SIG_BF16, binding.SIG_F16, binding.SIG_E4M3
OK, LARGE = binding.SIG_OK, binding.SIG_ERR_TOO_LARGE


@pytest.fixture(scope="module")
def launches(linked):   # noqa: F811
    """launches(calls): (status, most bytes asked for, launches) of each"""
    exe = linked("host_window_launches.cpp")

    def answers(calls):
        lines = run(exe, calls="".join(" ".join(str(word) for word in call) + "\n" for call in calls)).splitlines()
        assert len(lines) == len(calls)
        return [(int(line.split()[0]), int(line.split()[1]), [Launch(w) for w in line.split()[2:]]) for line in lines]

    return answers


HUGE = [(way, *shape) for way in ("forward", "backward")
        for shape in (((1 << 31) - 1, 1, 1, 1, 4, 4, BF16, 0, 0), (1, 1 << 30, 1, 1, 8, 8, F32, 100, 0), (1 << 22, 500, 8, 2, 8, 8, F16, 16, 3), (1, 1, 1 << 29, 1, 4, 4, F32, 0, 0))]
HUGE += [("append", 1 << 15, (1 << 16) - 1, 1, 1, 2, 2, BF16, cache, 16, 2) for cache in (BF16, E4M3)]
HUGE += [("append", (1 << 31) - 1, 1, 0, 1, 2, 2, F32, cache, 1, 0) for cache in (F32, E4M3)]
HUGE += [("attend", (1 << 31) - 1, 1, 1, 1, 4, 4, F32, F32, 16, 100, 0, 0), ("attend", 1, (1 << 31) - 1025, 1, 1, 4, 4, BF16, E4M3, 1 << 30, 2, 0, 0),
         ("attend", 1, 1, 1, 1, 256, 256, BF16, BF16, (1 << 31) - 1, (1 << 31) - 1, 0, 0)]


def test_no_launch_is_larger_than_launches_are(launches):
    for call, (rc, _, got) in zip(HUGE, launches(HUGE)):
        assert rc == OK and got, call
        for launch in got:
            assert within_limits(launch), (call, launch.kernel, launch.grid, launch.threads)


def test_what_no_launch_can_hold_is_refused(launches):
    calls = [("forward", 1 << 20, 1 << 25, 1, 1, 4, 4, F32, 0, 0), ("backward", 1, (1 << 31) - 1024, 1, 1, 4, 4, BF16, 0, 0),
             ("forward", 1, 1, (1 << 31) - 1, 1, 4, 4, F32, 0, 0), ("backward", 1, 1 << 20, 1 << 15, 1, 4, 4, F32, 0, 0),
             ("append", 1 << 16, 1 << 15, 1, 1, 2, 2, F32, F32, 16, 2),
             ("attend", 1 << 16, 1 << 20, 1, 1, 4, 4, F32, F32, 16, 100, 0, 0), ("attend", 1, 1, 1, 1, 4, 4, F32, F32, 1 << 32, 1, 0, 0)]
    for call, (rc, _, got) in zip(calls, launches(calls)):
        assert rc == LARGE and not got, (call, rc)


def test_every_query_and_key_has_a_workgroup(launches):
    """Queries: 128 a workgroup, 64 of more than 128 components, and of float32 from 65 on but for 96.  Keys: as many, cut along the queries or not."""
    for (B, T, H, G, K, V, kind), rows in (((3, 1000, 4, 2, 64, 64, BF16), 128), ((3, 1000, 4, 2, 64, 64, F32), 128), ((3, 1000, 4, 2, 96, 96, F32), 128), ((3, 1000, 4, 2, 96, 90, F32), 64), ((3, 1000, 4, 2, 128, 128, F32), 64), ((2, 129, 3, 3, 200, 16, F16), 64), ((700, 65, 2, 1, 30, 40, F16), 128)):
        ((rc, _, (forward,)), (rc2, _, backward)) = launches([("forward", B, T, H, G, K, V, kind, 10, 0), ("backward", B, T, H, G, K, V, kind, 10, 0)])
        tiles = -(-T // rows)
        assert rc == rc2 == OK and forward.workgroups == backward[0].workgroups == B * H * tiles
        assert "query_gradient" in backward[0].kernel and "key_gradient" in backward[1].kernel and backward[1].workgroups % (B * G * tiles) == 0


# B, T, heads, shared, window, sinks (64 components, bfloat16: 128 keys a workgroup): tiles that are cut, and parts.  256 compute units
CUT = [((4, 2048, 16, 4, 0, 0), (16, 2)),        # fewer than two a unit: two
       ((64, 2048, 16, 4, 0, 0), (0, 1)), ((8, 4096, 16, 16, 1024, 0), (0, 1)),
       ((8, 4096, 16, 16, 1024, 4), (1, 3)),     # the first tokens', whose queries are more than 2 (1,024 + 128)
       ((8, 4096, 16, 16, 1024, 129), (2, 3)), ((8, 2000, 16, 16, 1024, 4), (0, 1)), ((1, 65536, 16, 4, 1024, 4), (1, 30)), ((1, 1 << 20, 16, 4, 1024, 4), (1, 64)),
       ((256, 4096, 4, 4, 64, 1000), (0, 1)), ((256, 4096, 4, 1, 64, 1000), (8, 2)),      # 16 workgroups a unit at most, for the parts
       ((1, 100, 1, 1, 0, 0), (0, 1)),           # a part has 128 queries or more
       ((1, 300, 2, 2, 20, 0), (3, 2))]


def test_key_gradients_are_cut_by_their_rule(launches):
    got = launches([("backward", B, T, H, G, 64, 64, BF16, window, sinks) for (B, T, H, G, window, sinks), _ in CUT])
    for ((B, T, H, G, _, sinks), (cut, parts)), (rc, most, launched) in zip(CUT, got):
        tiles = -(-T // 128)
        assert rc == OK and launched[1].workgroups == B * G * (tiles - cut + cut * parts), (T, launched[1].workgroups)
        assert len(launched) == (3 if cut else 2)
        assert most == 4 * (B * H * T + cut * parts * B * G * 128 * 128), (T, most)


# B, T, heads, cache heads, page tokens, pages, window, sinks: parts of the places
SPLIT = [((128, 1, 4, 4, 16, 16, 0, 0), 1), ((32, 1, 32, 8, 64, 256, 0, 0), 2), ((1, 1, 16, 2, 64, 2048, 0, 0), 256), ((1, 1, 2, 2, 64, 2048, 500, 4), 3), ((1, 1, 1, 1, 16, 16, 0, 0), 1),
         ((1, 40, 16, 2, 64, 2048, 0, 0), 13), ((1, 1, 1, 1, 64, 1 << 20, 0, 0), 512)]


def test_places_are_cut_by_their_rule(launches):
    for cache in (BF16, E4M3):
        got = launches([("attend", B, T, H, G, 64, 64, BF16, cache, P, pages, window, sinks) for (B, T, H, G, P, pages, window, sinks), _ in SPLIT])
        for ((B, T, H, G, *_), splits), (rc, most, launched) in zip(SPLIT, got):
            tiles = -(-T * (H // G) // 16)
            assert rc == OK and launched[0].workgroups == B * G * tiles * splits and len(launched) == (2 if splits > 1 else 1)
            assert most == (4 * B * G * tiles * splits * 16 * 66 if splits > 1 else 0)


# B, T, heads, components, type, window, sinks: pieces of the keys (two workgroups a unit, pieces of 512 keys or more, or of 256 where workgroups are fewer than units)
PIECES = [((1, 4096, 1, 64, BF16, 0, 0), 16), ((1, 4096, 8, 64, BF16, 0, 0), 2), ((1, 65536, 1, 64, F32, 0, 0), 1), ((1, 32768, 1, 64, F16, 0, 0), 2), ((1, 4096, 1, 64, BF16, 300, 0), 1),
          ((1, 4096, 1, 64, BF16, 1000, 0), 4), ((1, 4096, 1, 64, BF16, 300, 2000), 9), ((1, 511, 1, 64, BF16, 0, 0), 1), ((1, 512, 1, 64, BF16, 0, 0), 2), ((16, 4096, 16, 64, BF16, 0, 0), 1),
          ((8, 512, 8, 64, BF16, 0, 0), 1), ((1, 8192, 3, 64, BF16, 0, 0), 3), ((1, 16384, 2, 256, F32, 0, 0), 1), ((1, 8192, 2, 200, F32, 0, 0), 2), ((1, 12000, 1, 16, BF16, 0, 0), 6)]


def test_queries_are_cut_along_their_keys_by_their_rule(launches):
    got = launches([(way, B, T, H, H, K, K, kind, window, sinks) for (B, T, H, K, kind, window, sinks), _ in PIECES for way in ("forward", "backward")])
    for i, ((B, T, H, K, kind, *_), splits) in enumerate(PIECES):
        (rc, most, forward), (rc2, _, backward) = got[2 * i:2 * i + 2]
        tiles = -(-T // (64 if K > 128 else 128))
        assert rc == rc2 == OK and forward[0].workgroups == backward[0].workgroups == B * H * tiles * splits, PIECES[i]
        assert len(forward) == (2 if splits > 1 else 1) and most == (4 * B * H * T * splits * (K + 2) if splits > 1 else 0)
        assert ("join_pieces" in backward[1].kernel) == (splits > 1)


def test_instances_by_size_and_type(launches):
    """Rows of 32, 64, 96, 128, 192 and 256 components; whole where keys and values have just that."""
    for dims, size, whole in (((32, 32), 32, 1), ((16, 32), 32, 0), ((33, 64), 64, 0), ((64, 64), 64, 1), ((96, 96), 96, 1), ((97, 5), 128, 0), ((128, 128), 128, 1), ((7, 150), 192, 0), ((192, 192), 192, 1), ((130, 256), 256, 0)):
        for kind in (F32, BF16, F16):
            ((rc, _, (forward,)),) = launches([("forward", 1, 10, 1, 1, *dims, kind, 0, 0)])
            found = re.search(r"Li(\d+)ELi(\d+)ELb([01])E", forward.kernel)
            assert rc == OK and (int(found.group(1)), int(found.group(3))) == (size, whole), (dims, forward.kernel)
