"""Region selection, region attention and dropout in 64 bits with numpy -- TEST INFRASTRUCTURE ONLY.

Written from the definitions in include/slide_attn.h, group by group; shares no code with the library.  `problem` is a dict:
heads, kv_heads, q_region, k_region, and optionally q_size, k_size (arrays [B, 2]), scale, dropout, seed, offset.
"""
import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def philox(c0, c1, c2, c3, seed, rounds=7):
    """Philox-4x32 of counters given as arrays (broadcast against each other); four uint64 arrays of 32-bit words."""
    c = [np.asarray(x, dtype=np.uint64) & M32 for x in (c0, c1, c2, c3)]
    c = [np.array(x) for x in np.broadcast_arrays(*c)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & M32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & M32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def _half(words, e):
    w = np.choose(np.asarray(e, dtype=np.int64) // 2, words)
    return (w >> (np.asarray(e, dtype=np.uint64) % np.uint64(2) * np.uint64(16))) & np.uint64(0xFFFF)


def _threshold(p):
    t = int(np.rint(np.float64(np.float32(p)) * 65536))
    return t, 65536.0 / (65536 - t)


def drop_factors(i, p, seed, offset):
    """The factors of the elements numbered i."""
    i = np.asarray(i, dtype=np.uint64)
    g = i >> np.uint64(3)
    words = philox(g, (g >> np.uint64(32)) | np.uint64(1 << 31), 0xFFFFFFFF, offset, seed)
    t, up = _threshold(p)
    return np.where(_half(words, i % np.uint64(8)) >= t, up, 0.0)


def weight_factors(p, seed, offset, bm, i, R, j, places):
    """The factors [R, places] of group (bm = b * kv_heads + m, i) and key region j."""
    r, n = np.arange(R)[:, None], np.arange(places)[None]
    words = philox(j * -(-places // 4) + n // 4, i * -(-R // 2) + r // 2, bm, offset, seed)
    t, up = _threshold(p)
    return np.where(_half(words, np.broadcast_to(4 * (r % 2) + n % 4, (R, places))) >= t, up, 0.0)


def regions(H, W, region):
    """For each region the list of its places' pixels, -1 outside the map."""
    h, w = min(region[0], H), min(region[1], W)
    found = []
    for y0 in range(0, H, h):
        for x0 in range(0, W, w):
            found.append([y * W + x if y < H and x < W else -1 for y in range(y0, y0 + h) for x in range(x0, x0 + w)])
    return np.array(found)


def _inside(size, b, H, W):
    ok = np.zeros((H, W), dtype=bool)
    h, w = (H, W) if size is None else (min(max(int(n), 0), m) for n, m in zip(size[b], (H, W)))
    ok[:h, :w] = True
    return np.append(ok.reshape(-1), False)             # [-1]: outside the map


def select(q, k, topk, problem):
    B, Hq, Wq, C = q.shape
    heads, kv = problem["heads"], problem.get("kv_heads") or problem["heads"]
    g, d = heads // kv, C // heads
    qr, kr = regions(Hq, Wq, problem["q_region"]), regions(k.shape[1], k.shape[2], problem["k_region"])
    index = np.full((B, kv, len(qr), topk), -1, dtype=np.int32)
    for b in range(B):
        q_in, k_in = _inside(problem.get("q_size"), b, Hq, Wq), _inside(problem.get("k_size"), b, k.shape[1], k.shape[2])
        qb, kb = q[b].reshape(-1, heads, d).astype(np.float64), k[b].reshape(-1, kv, d).astype(np.float64)
        for m in range(kv):
            K = [kb[p[k_in[p]], m] for p in kr]
            for i, p in enumerate(qr):
                p = p[q_in[p]]
                if len(p) == 0:
                    continue
                Q = qb[p, m * g:(m + 1) * g].sum((0, 1))
                s = [(-np.nan_to_num((Q * x.sum(0)).sum() / len(x), nan=-np.inf), j) for j, x in enumerate(K) if len(x)]
                chosen = sorted(j for _, j in sorted(s)[:topk])
                index[b, m, i, :len(chosen)] = chosen
    return index


def attention(q, k, v, index, problem, dout=None):
    """A dict of out, lse (dq, dk, dv), and of `out_mag`, `dq_mag`, ...: the same sums over absolute values, which bounds of
    rounding errors are made of."""
    B, Hq, Wq, C = q.shape
    Hk, Wk = k.shape[1:3]
    heads, kv = problem["heads"], problem.get("kv_heads") or problem["heads"]
    g, d = heads // kv, C // heads
    scale = problem.get("scale") or d ** -0.5
    p_drop = problem.get("dropout", 0.0)
    qr, kr = regions(Hq, Wq, problem["q_region"]), regions(Hk, Wk, problem["k_region"])
    R, J, places = qr.shape[1] * g, len(kr), kr.shape[1]
    Nq, Nk = Hq * Wq, Hk * Wk
    z = {n: np.zeros((B, Nq, heads, d)) for n in ("out", "out_mag", "dq", "dq_mag")}
    z.update({n: np.zeros((B, Nk, kv, d)) for n in ("dk", "dk_mag", "dv", "dv_mag")})
    z["lse"] = np.full((B, heads, Nq), -np.inf)
    z["score_mag"] = 0.0
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    for b in range(B):
        q_in, k_in = _inside(problem.get("q_size"), b, Hq, Wq), _inside(problem.get("k_size"), b, Hk, Wk)
        for m in range(kv):
            for i, qp in enumerate(qr):
                lists = [j for j in index[b, m, i] if 0 <= j < J]
                keys = np.concatenate([kr[j] for j in lists]) if lists else np.zeros(0, dtype=int)
                ok = k_in[keys]
                keys, rows_ok = keys[ok], q_in[qp]
                if not rows_ok.any() or len(keys) == 0:
                    continue
                px = qp[rows_ok]
                hs = slice(m * g, (m + 1) * g)
                Q = q[b].reshape(Nq, heads, d)[px, hs].reshape(-1, d)
                K, V = k[b].reshape(Nk, kv, d)[keys, m], v[b].reshape(Nk, kv, d)[keys, m]
                S = Q @ K.T * scale
                z["score_mag"] = max(z["score_mag"], (np.abs(Q) @ np.abs(K).T).max() * scale)
                top = S.max(1, keepdims=True)
                E = np.exp(S - top)
                P = E / E.sum(1, keepdims=True)
                lse = np.log(E.sum(1)) + top[:, 0]
                F = np.ones_like(P)
                if p_drop:
                    F = np.concatenate([weight_factors(p_drop, problem.get("seed", 0), problem.get("offset", 0), b * kv + m, i, R, int(j), places)
                                        for j in lists], 1)[:, ok]
                    F = F.reshape(len(qp), g, -1)[rows_ok].reshape(len(P), -1)
                O = (P * F) @ V
                fold = lambda x: x.reshape(len(px), g, *x.shape[1:])  # noqa: E731
                z["out"][b, px, hs] = fold(O)
                z["out_mag"][b, px, hs] = fold((P * F) @ np.abs(V))
                z["lse"][b, hs, px] = fold(lse)
                if dout is None:
                    continue
                dO = dout[b].reshape(Nq, heads, d).astype(np.float64)[px, hs].reshape(-1, d)
                D = (dO * O).sum(1, keepdims=True)
                dS = P * (F * (dO @ V.T) - D) * scale
                mag = P * (F * (np.abs(dO) @ np.abs(V).T) + 2 * (np.abs(dO) * np.abs(O)).sum(1, keepdims=True)) * scale
                z["dq"][b, px, hs] = fold(dS @ K)
                z["dq_mag"][b, px, hs] = fold(mag @ np.abs(K))
                np.add.at(z["dk"][b, :, m], keys, dS.T @ Q)
                np.add.at(z["dk_mag"][b, :, m], keys, mag.T @ np.abs(Q))
                np.add.at(z["dv"][b, :, m], keys, (P * F).T @ dO)
                np.add.at(z["dv_mag"][b, :, m], keys, (P * F).T @ np.abs(dO))
    for n in z:
        if n in ("out", "out_mag", "dq", "dq_mag"):
            z[n] = z[n].reshape(B, Hq, Wq, heads * d)
        elif n.startswith(("dk", "dv")):
            z[n] = z[n].reshape(B, Hk, Wk, kv * d)
    z["lse"] = z["lse"].reshape(B, heads, Hq, Wq)
    return z
