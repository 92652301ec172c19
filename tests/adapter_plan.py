"""Into how many parts the adapters' gradient kernel cuts each adapter: the planning rule of ep_adapters.cu once more, so that tests can tell
which cases reach the sums of several parts."""
import numpy as np


def parts(offsets, entries, H, N, rank, down=True, up=True):
    """Parts of each adapter (0: no entries) in a call for ddown (down) and dup (up)."""
    f32, per_stage, ctas_most = np.float32, 64, 2 * 148
    A, (tiles_h, tiles_n) = len(offsets) - 1, [-(-c // 128) for c in (H, N)]
    stages = [-(-(int(offsets[a + 1]) - int(offsets[a])) // per_stage) for a in range(A)]
    full = entries // per_stage
    least = max(8, -(-(full * (tiles_h + tiles_n)) // (3 * ctas_most)))
    ctas = min((A + full // least) * (tiles_h + tiles_n), ctas_most if rank <= 64 else ctas_most // 2)
    tiles = tiles_h * down + tiles_n * up
    longest, best = max(stages), None
    for cut in (1, 2, 3, 4, 6, 8, 12, 16):
        piece = max(least, -(-longest // cut))
        split = sum(-(-n // piece) for n in stages if n > piece)
        share = (f32(sum(stages)) + f32(5) * f32(split)) * f32(tiles) / f32(ctas)
        cost = max(f32(0.6) * f32(min(piece, longest)), share) + f32(8 if split else 0)
        if best is None or cost < best[0]:
            best = (cost, piece)
    return [-(-n // best[1]) for n in stages]
