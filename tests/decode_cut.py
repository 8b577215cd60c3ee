"""How st3_block_decode cuts a call, told from sizes alone: what a test expects its sizes to reach.  test_decode_cuts.py holds it against the workspaces
that the library asks for, so that a changed rule is noticed there."""

BLOCK, COLS, WAVE, LDS = 64, 16, 64, 160 << 10
WHOLE_STRIPS, SHORT_UNITS, MANY_STRIPS, STAGE_BYTES, CHUNK_WGS = 192, 20, 256, 20 << 10, 768


def attend_lds(d, waves, cols, staged_rows):
    return max(waves * BLOCK * d, 4 * waves * cols * (d + 4)) + 4 * (2 * waves * COLS + 2 * COLS + cols * staged_rows)


def cut(batch, heads, kv_heads, d, max_len, scored):
    """(waves of a workgroup, blocks of a chunk, chunks that there is room for); no blocks: whole strips, one launch."""
    G = heads // kv_heads
    shared, cols = -(-G // COLS), min(G, COLS)
    units, strips = max_len // BLOCK + 1, batch * kv_heads * shared
    waves = 4 if strips > MANY_STRIPS else 12
    fits = units + 2 <= waves * WAVE and (not scored or (shared == 1 and attend_lds(d, waves, cols, units * BLOCK) <= LDS))
    if fits and (strips >= WHOLE_STRIPS or units <= SHORT_UNITS):
        return waves, 0, 0
    top = 4 * WAVE - 2
    if scored:
        top = min(top, max(8, STAGE_BYTES // (cols * BLOCK * 4)))
    chunk = min(max(4, -(-units * strips // CHUNK_WGS)), top, units)
    most = max(min(-(-units // 4), -(-CHUNK_WGS // strips)), -(-units // top))
    return 4, chunk, most


def workspace(batch, heads, kv_heads, d, max_len):
    up = lambda n: -(-n // 256) * 256
    need = 256
    for scored in (False, True):
        _, chunk, most = cut(batch, heads, kv_heads, d, max_len, scored)
        if chunk:
            rows = batch * heads
            need = max(need, up(rows * most * d * 4) + up(rows * most * 8) + (up(rows * (max_len // BLOCK + 1) * BLOCK * 4) if scored else 0))
    return need
