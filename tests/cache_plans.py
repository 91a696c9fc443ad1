"""How the library splits a cache call over CTAs, worked out again from the sizes: tests name the split they
mean to reach and assert that they reach it."""


def stages(dim):
    return 6 if dim == 256 else 3


def attend_split(lens, heads, dim, max_len, scored, masked, sms=148):
    """{"cluster": CTAs per row, "each": tiles of a CTA} or {"cluster": 0, "each", "with_rows", "parts": per non-empty row, if shares
    end with rows}.  (At 256 channels: as long as the rows' clusters fit the GPU at once.)"""
    up = lambda a, b: -(-a // b)
    tile = 8192 // dim
    rows, row_tiles, limit = len(lens) * heads, up(max_len, tile), sms * (1 if dim == 256 else 2)
    most, size = 8 if dim == 256 else 16, 1
    while size < most and size < row_tiles and rows * size * 2 <= sms:
        size *= 2
    many = rows * 2 > limit
    if row_tiles <= size * (16 if many else 6) and (many or not scored):
        return {"cluster": size, "each": up(up(max(lens), tile), size)}
    grid = min(limit, rows * row_tiles)
    tiles = [up(n, tile) for n in lens]
    each = max(1, up(sum(tiles) * heads, grid))
    if each >= 6 and not masked:
        for k in range(4):
            e = each + k * (each // 6) // 3
            if sum(up(t, e) for t in tiles) * heads <= grid:
                return {"cluster": 0, "each": e, "with_rows": True, "parts": sorted({up(t, e) for t in tiles if t})}
    return {"cluster": 0, "each": each, "with_rows": False}


def select_split(rows, max_len, sms=148):
    """(CTAs per row, keys per thread that the kernel is built for; 0: keys read again for every step)"""
    size = 1
    while size < 8 and (size * 1024 * 33 < max_len or (rows * size * 2 <= sms and size * 1024 * 3 < max_len)):
        size *= 2
    per = -(-max_len // (size * 1024))
    return size, next((k for k in (3, 9, 17, 25, 33) if per <= k), 0)
