"""The scratch that window attention and attention over a cache ask for, against the bounds that include/sig_sequence.h states, on the CPU (256 compute units)."""
import random

from test_host_window_launches import BF16, F16, F32, OK, launches      # noqa: F401 (a fixture)
from test_host_sanitized import linked      # noqa: F401 (a fixture)

UNITS = 256


def rows_of(kind, K, V):
    """queries or keys of a workgroup"""
    return 64 if (kind != F32 and max(K, V) > 128) or (kind == F32 and max(K, V) > 64 and not K == V == 96) else 128


def test_no_call_asks_for_more_than_the_header_says(launches):   # noqa: F811
    rng = random.Random(3)
    sizes = [16, 40, 64, 72, 96, 128, 192, 256]
    windows, caches = [], []
    # (511 workgroups of queries: two pieces each, almost four workgroups' pieces a unit)
    windows += [(511, 100, 1, 1, 64, 64, BF16, 0, 0), (7, 128 * 73, 1, 1, 64, 64, BF16, 0, 0), (1, 8192, 3, 3, 64, 64, BF16, 0, 0)]
    caches += [(511, 1, 1, 1, 64, 64, BF16, BF16, 64, 64, 0, 0), (1, 40, 16, 2, 64, 64, BF16, BF16, 64, 2048, 0, 0)]
    for _ in range(400):
        G = rng.choice((1, 2, 3, 8))
        H, K = G * rng.choice((1, 2, 4)), rng.choice(sizes)
        V, kind = rng.choice((K, K, rng.choice(sizes))), rng.choice((F32, BF16, F16))
        B, T = int(2 ** rng.uniform(0, 9.5)), int(2 ** rng.uniform(0, 16))
        window, sinks = rng.choice((0, int(2 ** rng.uniform(0, 13)))), rng.choice((0, 1, 70, 1000))
        windows.append((B, T, H, G, K, V, kind, window, sinks))
        caches.append((B, int(2 ** rng.uniform(0, 8)), H, G, K, V, kind, kind, rng.choice((8, 16, 64)), int(2 ** rng.uniform(0, 12)), window, sinks))
    got = launches([(way, *call) for call in windows for way in ("forward", "backward")])
    largest = 0
    for i, (B, T, H, G, K, V, kind, window, sinks) in enumerate(windows):
        (rc, forward, _), (rc2, backward, _) = got[2 * i:2 * i + 2]
        rows = rows_of(kind, K, V)
        assert rc == rc2 == OK
        assert forward < 4 * 4 * UNITS * rows * (V + 2), windows[i]
        largest = max(largest, forward / (4 * UNITS * rows * (V + 2)))
        # the queries' pieces; the first tokens' parts; all keys' parts
        assert backward <= 4 * (B * H * T + max(4 * UNITS * rows * K, 16 * UNITS * rows * (K + V) if sinks else 4 * UNITS * rows * (K + V))), windows[i]
    assert largest > 3      # (not two)
    largest = 0
    for call, (rc, most, _) in zip(caches, launches([("attend", *call) for call in caches])):
        V = call[5]
        assert rc == OK and most < 4 * 4 * UNITS * 16 * (V + 2), call
        largest = max(largest, most / (4 * UNITS * 16 * (V + 2)))
    assert largest > 3
