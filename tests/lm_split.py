"""The selective scan's split of its steps, as lm_select.hpp has it: tests that mean to meet a composition of pieces assert that they do."""
TILE, COLUMNS, LEAST_TILES, MOST_SPANS, MAPS_AT_ONCE = 16, 64, 2, 256, 1536
FORWARD_AT_ONCE, GRADIENT_AT_ONCE = 1024, 512


def _over(a, b):
    return -(-a // b)


def split(B, T, D, at_once):
    """(spans, pieces of a span, tiles of a span, tiles of a piece)"""
    groups, tiles = B * _over(D, COLUMNS), _over(T, TILE)
    best, least, spans = 1, 4 * _over(groups, at_once) * tiles, 2
    while spans <= MOST_SPANS and spans * LEAST_TILES <= tiles and groups < 8 * at_once:
        each = _over(tiles, spans)
        cost = 4 * _over(groups * spans, at_once) * each + _over(groups * (spans - 1), at_once) * each + spans // 4
        if cost < least:
            best, least = spans, cost
        spans += 1
    each = _over(tiles, best)
    spans = _over(tiles, each)
    parts = MAPS_AT_ONCE // (groups * (spans - 1)) if spans > 1 else 1
    parts = max(1, min(parts, each // LEAST_TILES))
    piece = _over(each, parts)
    return spans, _over(each, piece), each, piece


def empty_pieces(T, spans, parts, each, piece):
    """Pieces of the last span that no step is left for."""
    left = _over(T, TILE) - (spans - 1) * each
    return parts - _over(left, piece)


def workspaces(B, T, D, N):
    """Bytes that the split asks for, forward and backward."""
    up = lambda n: -(-n // 16) * 16
    spans, parts, _, _ = split(B, T, D, FORWARD_AT_ONCE)
    forward = B * spans * parts * D * (N + 1) * 4 if spans > 1 else 0
    spans, parts, _, _ = split(B, T, D, GRADIENT_AT_ONCE)
    maps = up(B * spans * parts * D * N * 4) + up(B * spans * parts * D * 4) if spans > 1 else 0
    return forward, maps + up(_over(D, COLUMNS) * B * T * 2 * N * 4) + B * spans * D * (N + 2) * 4
