"""How lookm_chunk_attention and lookm_step_attention divide a call's work among the SMs, restated, so that a test can say which plan its
sizes get.  The number of launches tells whether the library took shares; sets of one or of two query tiles leave no trace outside."""
TILE, MANY, MOST_CTAS = 128, 128, 192


def ceil(a, b):
    return -(-a // b)


def unit_steps(n_new, length, set_no, set_tiles, tile_tokens):
    """(steps, tiles of cached rows, whether it is a pair)"""
    tok0 = set_no * set_tiles * tile_tokens
    pair = set_tiles == 2 and tok0 + tile_tokens < n_new
    last = min(n_new, tok0 + (2 if pair else 1) * tile_tokens)
    tiles = ceil(length - n_new + last, TILE)
    return 2 + (2 if pair else 1) * tiles, tiles, pair


def entries(reqs, tile_tokens, set_tiles):
    """Sets of query tiles, in the order in which they are dealt: a list per entry, the last set (the first that is dealt) at the end."""
    sets = [ceil(ceil(n, tile_tokens), set_tiles) for n, _ in reqs]
    each = len(reqs) > 1 and sum(sets) <= MANY
    out = []
    for (n, length), k in zip(reqs, sets):
        units = [unit_steps(n, length, s, set_tiles, tile_tokens) for s in range(k)]
        out += [[u] for u in units] if each else [units]
    return sorted(out, key=lambda e: -e[-1][0])


def deal(es, heads, sms):
    """Steps of all units and of the SM that has most; that is 0 for so many units that they even out."""
    if sum(map(len, es)) * heads >= 4 * sms:
        return 0, 0
    load, i, step = [0] * sms, 0, 1
    for e in es:
        for u in reversed(e):
            for _ in range(heads):
                load[i] += u[0]
                i += step
                if i in (-1, sms):
                    i, step = i - step, -step
    return sum(load), max(load)


def in_shares(total, rows, sms):
    return ceil(total, sms) + 8 + rows // 8


class Plan:
    """set_tiles: query tiles of a set.  launches: of each, whether it is in shares, its whole units, those that are pairs, the steps of the
    longest unit and of a share."""

    def __init__(self, new, lens, hq, hkv, page, sms):
        sms, group = min(sms, MOST_CTAS), hq // hkv
        tile_tokens = TILE // group
        reqs = [(n, length) for n, length in zip(new, lens) if n]
        most_new = max(new)
        rows = min(2 * tile_tokens * group, max(most_new, 1) * group)
        es, self.set_tiles = entries(reqs, tile_tokens, 2), 2
        if most_new > tile_tokens and len(es) <= MANY:
            total2, most2 = deal(es, hkv, sms)
            ones = entries(reqs, tile_tokens, 1)
            if most2 and len(ones) <= MANY:
                total1, most1 = deal(ones, hkv, sms)
                a, b = min(most1, in_shares(total1, min(rows, TILE), sms)), min(most2, in_shares(total2, rows, sms))
                if most1 and (33 if page == 16 else 26) * a < 20 * b:
                    es, self.set_tiles = ones, 1
        if self.set_tiles == 1:
            rows = min(rows, TILE)
        self.loaders = 2 if page == 16 and most_new <= tile_tokens else 1
        self.launches = []
        for i in range(0, len(es), MANY):
            part = es[i:i + MANY]
            total, most = deal(part, hkv, sms)
            units = [u for e in part for u in e]
            self.launches.append(dict(shares=most > in_shares(total, rows, sms) if most else False, units=len(units) * hkv,
                                      pairs=sum(u[2] for u in units) * hkv, longest=max(u[0] for u in units), share=ceil(total, sms) if total else 0))

    def n_launches(self, step=False, longest=0):
        """Kernels that the call enqueues.  Steps on caches of up to 2048 rows add their weights in the first launch."""
        return sum(2 if x["shares"] or (step and longest > 2048) else 1 for x in self.launches)
