"""The 4-bit key/value cache in plain numpy: rows quantised by the definition in
binary32, everything else in 64 bits, one row at a time."""
import numpy as np


def bf16(x):
    """float32 -> bf16 bits, nearest-even, as float32."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = (u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16
    return r.astype(np.uint32).view(np.float32)


def quantise(x):
    """Rows x (..., D) float32 -> (codes, s, z); s NaN where a row cannot be held."""
    x = np.asarray(x, np.float32)
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    fine = np.isfinite(x).all(-1, keepdims=True)
    with np.errstate(all="ignore"):
        u = lo.view(np.uint32).astype(np.uint64)
        z = ((np.where(u >> 31, u + 0xFFFF, u) & 0xFFFF0000).astype(np.uint32)).view(np.float32)
        q = (hi - z) / np.float32(15)
        u = q.view(np.uint32).astype(np.uint64)
        s = (((u + 0xFFFF) & 0xFFFF0000).astype(np.uint32)).view(np.float32)
        bad = ~fine | ~np.isfinite(z) | ~np.isfinite(s)
        c = np.where(s > 0, np.clip(np.rint((x - z) / s), 0, 15), 0)
    c = np.where(bad, 0, c)
    return c, np.where(bad, np.nan, s).astype(np.float32), np.where(bad, 0, z).astype(np.float32)


def held(x):
    c, s, z = quantise(x)
    return z.astype(np.float64) + s.astype(np.float64) * c


class Cache:
    def __init__(self, n_slots, H, D, cap):
        self.H, self.D, self.cap = H, D, cap
        self.k = [np.zeros((H, 0, D)) for _ in range(n_slots)]
        self.v = [np.zeros((H, 0, D)) for _ in range(n_slots)]
        self.pos = [np.zeros((H, 0), np.int64) for _ in range(n_slots)]
        self.w = [np.zeros((H, 0)) for _ in range(n_slots)]
        self.next = [0] * n_slots

    def named(self, slots, B):
        ids = range(B) if slots is None else slots
        return [(b, s) for b, s in enumerate(ids) if 0 <= s < len(self.k)]

    def rows(self, b, N, nodes, count):
        if count is None:
            return list(range(N))
        n = int(count[b])
        if nodes is None:
            return list(range(min(max(n, 0), N)))
        got = [0]
        for i in nodes[b][:min(max(n, 0), N - 1)]:
            if not 0 <= i < N:
                break
            got.append(int(i))
        return got

    def reset(self, slots=None):
        for s in range(len(self.k)) if slots is None else [s for s in slots if 0 <= s < len(self.k)]:
            self.k[s], self.v[s] = self.k[s][:, :0], self.v[s][:, :0]
            self.pos[s], self.w[s], self.next[s] = self.pos[s][:, :0], self.w[s][:, :0], 0

    def append(self, k, v, nodes=None, count=None, weight=None, slots=None):
        """k, v (B, N, H, D) float32."""
        B, N = k.shape[:2]
        for b, s in self.named(slots, B):
            rows = self.rows(b, N, nodes, count)
            fit = rows[:self.cap - self.k[s].shape[1]]
            self.k[s] = np.concatenate([self.k[s], held(k[b, fit].transpose(1, 0, 2))], 1)
            self.v[s] = np.concatenate([self.v[s], held(v[b, fit].transpose(1, 0, 2))], 1)
            at = self.next[s] + np.arange(len(fit))
            self.pos[s] = np.concatenate([self.pos[s], np.broadcast_to(at, (self.H, len(fit)))], 1)
            w = np.zeros((self.H, len(fit))) if weight is None else weight[b][:, fit]
            self.w[s] = np.concatenate([self.w[s], w], 1)
            self.next[s] += len(rows)

    def attend(self, q, k=None, v=None, n_nodes=None, mask=None, scale=1.0, slots=None):
        """-> out, lse and the bounds that their errors are derived from: the
        largest sum of |q k| of a row's scores, and sum p |v|."""
        B, N, Hq, D = q.shape
        G = Hq // self.H
        out, spread = np.zeros((B, N, Hq, D)), np.zeros((B, N, Hq, D))
        lse, size = np.full((B, N, Hq), -np.inf), np.zeros((B, N, Hq))
        for b, s in self.named(slots, B):
            m = N if n_nodes is None else min(max(int(n_nodes[b]), 0), N)
            for i in range(m):
                if k is None:
                    seen = []
                elif mask is None:
                    seen = list(range(i + 1))
                else:
                    seen = [u for u in range(m) if (int(mask[b, i, u // 32]) >> (u % 32)) & 1]
                for h in range(self.H):
                    K, V = self.k[s][h], self.v[s][h]
                    if seen:
                        K = np.concatenate([K, k[b, seen, h].astype(np.float64)])
                        V = np.concatenate([V, v[b, seen, h].astype(np.float64)])
                    if not len(K):
                        continue
                    for a in range(h * G, h * G + G):
                        x = q[b, i, a].astype(np.float64)
                        with np.errstate(all="ignore"):
                            S = scale * (K @ x)
                            top = S.max()
                            e = np.exp(S - top)
                            p = e / e.sum()
                            out[b, i, a], lse[b, i, a] = p @ V, top + np.log(e.sum())
                            size[b, i, a] = abs(scale) * (np.abs(K) @ np.abs(x)).max()
                            spread[b, i, a] = p @ np.abs(V)
        return out, lse, size, spread

    def weigh(self, q, lse, nodes=None, count=None, scale=1.0, slots=None):
        B, N, Hq, D = q.shape
        G = Hq // self.H
        for b, s in self.named(slots, B):
            for i in self.rows(b, N, nodes, count):
                for a in range(Hq):
                    l = float(lse[b, i, a])
                    if l != -np.inf:
                        x = q[b, i, a].astype(np.float64)
                        self.w[s][a // G] += np.exp(scale * (self.k[s][a // G] @ x) - l)

    def evict(self, keep, recent, slots=None, B=None):
        for b, s in self.named(slots, len(self.k) if B is None else B):
            n = self.k[s].shape[1]
            if n <= keep:
                continue
            for x in (self.k, self.v, self.pos, self.w):
                x[s] = x[s].copy()
            for h in range(self.H):
                young = self.pos[s][h] >= self.next[s] - recent
                w = self.w[s][h]
                rank = sorted(range(n), key=lambda j: (not young[j], w[j] != w[j], 0 if w[j] != w[j] else -w[j], j)
                              if not young[j] else (False, False, 0, j))
                kept = set(rank[:keep])
                late = [j for j in range(keep, n) if j in kept]
                for hole, j in zip([j for j in range(keep) if j not in kept], late):
                    for x in (self.k, self.v, self.pos, self.w):
                        x[s][h, hole] = x[s][h, j]
            for x in (self.k, self.v, self.pos, self.w):
                x[s] = x[s][:, :keep]
