"""Plain 64-bit definitions of integer attention over a cache of blocks: block tables and slots, rotary positions with the cache
in 8 bits, and the attention. NumPy and Python integers only."""
import numpy as np

BLOCK = 128


def blocks_of(tokens):
    return -(-tokens // BLOCK)


def plan(held, add, table, ring, state, rows):
    """(held_out, row_start, slot, position, state_out, refused); table and ring are changed in place."""
    width, size = table.shape[1], len(ring)
    head, count = int(state[0]), int(state[1])
    held_out, start = [], [0]
    slot, position = np.full(rows, -1, np.int64), np.zeros(rows, np.int64)
    taken = asked = refused = 0
    given = []
    for q, (h, a) in enumerate(zip(held, add)):
        h, a = int(h), int(a)
        sane, grow, at = 0 <= h <= width * BLOCK and a >= -1, max(a, 0), start[-1]
        start.append(at + grow)
        if sane and a == -1:
            given += table[q][:blocks_of(h)].tolist()
            held_out.append(0)
            continue
        need = blocks_of(h + grow) - blocks_of(h)
        ok = sane and blocks_of(h + grow) <= width and at + grow <= rows
        if ok:
            asked += need
            ok = need == 0 or asked <= count
        refused += not ok
        if ok:
            for c in range(blocks_of(h), blocks_of(h + grow)):
                table[q][c] = ring[(head + taken) % size]
                taken += 1
        held_out.append(h + grow if ok else h)
        for r in range(at, min(at + grow, rows)):
            p = h + r - at
            position[r] = p
            if ok:
                slot[r] = int(table[q][p // BLOCK]) * BLOCK + p % BLOCK
    for i, b in enumerate(given):
        ring[(head + count + i) % size] = b
    return (np.array(held_out, np.int64), np.minimum(start, rows), slot, position,
            np.array([(head + taken) % size, count - taken + len(given)]), refused)


def rotated(x, position, table, rot, layout):
    """x int64 [rows, heads, dim]; table int [positions, rot / 2, 2] in units of 2^-14."""
    x = np.clip(x, -32768, 32767).astype(np.int64)
    if not rot:
        return x
    i = np.arange(rot // 2)
    lo, hi = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    cs = table.astype(np.int64)[np.clip(position, 0, len(table) - 1)][:, None]
    a, b, c, s = x[..., lo], x[..., hi], cs[..., 0], cs[..., 1]
    x[..., lo], x[..., hi] = (a * c - b * s + 8192) >> 14, (a * s + b * c + 8192) >> 14
    return x


def exponent(amax, headroom):
    e = 0
    while int(amax) * (8 + headroom) > 1016 << e:
        e += 1
    return e


def eight_bits(x, e):
    return np.clip((x + ((1 << e) >> 1)) >> e, -127, 127).astype(np.int8)


def append(desc, q, k, v, slot, position, cache):
    """(q8, q_exp); the cache (dict of arrays) is changed in place."""
    heads, kv, dim = desc["heads"], desc["kv_heads"], desc["head_dim"]
    ro, (kh, vh) = desc.get("rotary") or {"table": None, "dim": 0, "layout": "half"}, desc.get("headroom", (0, 0))
    rows = len(slot)
    turn = lambda x, n: rotated(x.reshape(rows, n, dim).astype(np.int64), position, ro["table"], ro["dim"], ro["layout"])   # noqa: E731
    q, k = turn(q, heads), turn(k, kv)
    v = np.clip(v.reshape(rows, kv, dim).astype(np.int64), -32768, 32767)
    q8, q_exp = np.zeros((rows, heads, dim), np.int8), np.zeros((rows, heads), np.uint8)
    for r in range(rows):
        for h in range(heads):
            q_exp[r, h] = exponent(np.abs(q[r, h]).max(), 0)
            q8[r, h] = eight_bits(q[r, h], int(q_exp[r, h]))
    for r in range(rows):                                      # a block's first token decides
        if slot[r] >= 0 and slot[r] % BLOCK == 0:
            for h in range(kv):
                cache["k_exp"][slot[r] // BLOCK, h] = exponent(np.abs(k[r, h]).max(), kh)
                cache["v_exp"][slot[r] // BLOCK, h] = exponent(np.abs(v[r, h]).max(), vh)
    for r in range(rows):
        b, off = divmod(int(slot[r]), BLOCK)
        for h in range(kv if slot[r] >= 0 else 0):
            cache["k"][b, h, off] = eight_bits(k[r, h], min(12, int(cache["k_exp"][b, h])))
            cache["v"][b, h, :, off] = eight_bits(v[r, h], min(12, int(cache["v_exp"][b, h])))
    return q8, q_exp


def _segments():
    out = []
    for c in range(64):                                        # 2^(23 + (2 c + 1) / 128) to the nearest whole number
        x = 1 << 23
        for bit in range(22, -1, -1):
            if (2 * (x + (1 << bit)) - 1) ** 128 <= 1 << (128 * 24 + 2 * c + 1):
                x += 1 << bit
        out.append(max(1 << 23, x - 65536))
    return np.array(out, np.int64)


SEGMENTS = _segments()


def weight(n):
    """2^(15 + n / 2^13), n <= 0, rounded to nearest even."""
    n = np.maximum(n, -(1 << 18))
    g = n & 8191
    m, drop = SEGMENTS[g >> 7] + 1024 * (g & 127), 8 - (n >> 13)
    whole, rest, half = m >> drop, m & ((np.int64(1) << drop) - 1), np.int64(1) << (drop - 1)
    return whole + ((rest > half) | ((rest == half) & (whole % 2 == 1)))


def _scaled(x, n):
    return x << n if n >= 0 else x >> -n


def outputs(A, L, V, m0, s, clamp):
    """One row's head: Python integers."""
    y = []
    a = 32 - int(L).bit_length()
    rho = ((1 << 63) - 1) // _scaled(int(L), a) if L else 0
    for A_d, m, sh in zip(A.tolist(), m0.tolist(), s.tolist()):
        o = (_scaled(A_d, a - 8) * rho + (1 << (46 - V))) >> (47 - V) if L else 0
        v = (o * m + (1 << (30 + sh))) >> (31 + sh)
        y.append(min(max(v, clamp[0]), clamp[1]) if clamp else min(max(v, -2 ** 31), 2 ** 31 - 1))
    return y


def seen(desc, held, position):
    """The keys that a row sees, as a boolean array of `held`."""
    t = np.arange(held)
    keep = np.ones(held, bool)
    if desc.get("causal", True):
        keep &= t <= position
    if desc.get("window", 0):
        keep &= t > position - desc["window"]
    return keep


def forward(desc, q8, q_exp, row_start, held, table, cache, y):
    """y [rows, heads * dim] int64 is changed in place where a request has rows."""
    heads, kv, dim = desc["heads"], desc["kv_heads"], desc["head_dim"]
    group, (sm, ss), out = heads // kv, desc["score"], desc["out"]
    m0, s = (np.asarray(out[k], np.int64).reshape(heads, dim) for k in ("m0", "s"))
    for q in range(len(held)):
        total = min(max(int(held[q]), 0), table.shape[1] * BLOCK)
        ids = np.asarray(table[q][:blocks_of(total)], np.int64)
        good = np.repeat((ids >= 0) & (ids < len(cache["k"])), BLOCK)[:total]
        ids = np.clip(ids, 0, len(cache["k"]) - 1)
        for h in range(kv):
            k = cache["k"][ids, h].reshape(-1, dim)[:total].astype(np.int64)
            v = cache["v"][ids, h].transpose(0, 2, 1).reshape(-1, dim)[:total].astype(np.int64)
            ek, ev = (np.repeat(np.minimum(cache[x][ids, h].astype(np.int64), 12), BLOCK)[:total] for x in ("k_exp", "v_exp"))
            for r in range(int(row_start[q]), int(row_start[q + 1])):
                keep = seen(desc, total, total - int(row_start[q + 1]) + r) & good
                for g in range(h * group, (h + 1) * group):
                    A, L, V = np.zeros(dim, np.int64), 0, 0
                    if keep.any():
                        e = min(int(q_exp[r, g]), 12) + ek
                        W = np.minimum((np.int64(sm) << e) >> ss, 2 ** 31 - 1)
                        t = ((k @ q8[r, g].astype(np.int64)) * W) >> 23
                        V = int(ev[keep].max())
                        p = np.where(keep, weight(np.where(keep, t - t[keep].max() - 8192 * (V - ev), 0)), 0)
                        A, L = p @ v, int((p << np.where(keep, V - ev, 0)).sum())
                    y[r, g * dim:(g + 1) * dim] = outputs(A, L, V, m0[g], s[g], out.get("clamp"))
    return y
