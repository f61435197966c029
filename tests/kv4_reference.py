"""A plain statement of the paged 4-bit KV cache in numpy: the quantiser by nearest value from tables (float64), the maps by
lists, attention by the textbook formula in float64.  Shares no code with the library."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127], np.float64)


def nearest(x, table):
    """Index of the nearest entry of an ascending table, ties to the even index, saturating."""
    hi = np.clip(np.searchsorted(table, x), 1, len(table) - 1)
    up, down = table[hi] - x, x - table[hi - 1]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)


def stored(x, exp):
    """What the cache holds for x [n, Hkv, d] (float64) under exponents exp [Hkv]."""
    n, h, d = x.shape
    one = 2.0 ** np.asarray(exp, np.float64)[None, :, None, None]
    b = np.where(np.isnan(x), 0.0, x).reshape(n, h, d // 16, 16) / one
    s = E4M3[nearest(np.minimum(np.abs(b).max(-1, keepdims=True) / 6, 1e6), E4M3)]
    y = np.divide(np.minimum(np.abs(b), 1e30), s, out=np.zeros_like(b), where=s > 0)
    return (np.sign(b) * E2M1[nearest(np.minimum(y, 100.0), E2M1)] * s * one).reshape(n, h, d)


class Cache:
    """refs / table / lens as the library is to leave them, and for each (page, slot) what it holds: K, V [n_pages, ps, Hkv, d]."""

    def __init__(self, n_seqs, max_pages, n_pages, Hkv, d, ps, k_exp=None, v_exp=None):
        self.n, self.mp, self.np, self.ps = n_seqs, max_pages, n_pages, ps
        self.k_exp = [0] * Hkv if k_exp is None else k_exp
        self.v_exp = [0] * Hkv if v_exp is None else v_exp
        self.refs = np.zeros(n_pages, np.int64)
        self.table = np.full((n_seqs, max_pages), -1, np.int64)
        self.lens = np.zeros(n_seqs, np.int64)
        self.K = np.zeros((n_pages, ps, Hkv, d))
        self.V = np.zeros((n_pages, ps, Hkv, d))

    def pages(self, n):
        return -(-int(n) // self.ps)

    def rows(self, i):
        t = np.arange(self.lens[i])
        return self.table[i, t // self.ps], t % self.ps

    def kv(self, i):
        p, s = self.rows(i)
        return self.K[p, s], self.V[p, s]

    def append(self, k, v, cu):
        """k, v float64 [T, Hkv, d].  Returns False, with nothing changed, where pages or room are missing."""
        need = []
        for i in range(self.n):
            add, L = int(cu[i + 1] - cu[i]), int(self.lens[i])
            if self.pages(L + add) > self.mp:
                return False
            cow = add > 0 and L % self.ps and self.refs[self.table[i, L // self.ps]] > 1
            need.append((self.pages(L + add) - self.pages(L) + bool(cow), bool(cow)))
        free = [p for p in range(self.np) if self.refs[p] == 0]
        if sum(a for a, _ in need) > len(free):
            return False
        sk, sv = stored(k, self.k_exp), stored(v, self.v_exp)
        gone = []
        for i in range(self.n):
            add, L = int(cu[i + 1] - cu[i]), int(self.lens[i])
            mine, free = free[:need[i][0]], free[need[i][0]:]
            self.refs[mine] = 1
            if need[i][1]:
                at, fresh = L // self.ps, mine.pop(0)
                old = self.table[i, at]
                gone.append(old)
                self.K[fresh, :L % self.ps], self.V[fresh, :L % self.ps] = self.K[old, :L % self.ps], self.V[old, :L % self.ps]
                self.table[i, at] = fresh
            self.table[i, self.pages(L):self.pages(L) + len(mine)] = mine
            self.lens[i] = L + add
            for j in range(add):
                p, s = self.table[i, (L + j) // self.ps], (L + j) % self.ps
                self.K[p, s], self.V[p, s] = sk[cu[i] + j], sv[cu[i] + j]
        for p in gone:
            self.refs[p] -= 1
        return True

    def fork(self, parent):
        old_table, old_lens = self.table.copy(), self.lens.copy()
        for i in range(self.n):
            for p in old_table[i, :self.pages(old_lens[i])]:
                self.refs[p] -= 1
            self.lens[i] = 0 if parent[i] < 0 else old_lens[parent[i]]
            n = self.pages(self.lens[i])
            if n:
                self.table[i, :n] = old_table[parent[i], :n]
            for p in self.table[i, :n]:
                self.refs[p] += 1

    def compact(self, keep):
        plans, need = [], 0
        for i in range(self.n):
            L = int(self.lens[i])
            k = np.flatnonzero(keep[i, :L])
            holes = np.flatnonzero(keep[i, :L] == 0)
            stay = self.pages(L) if len(holes) == 0 else int(holes[0]) // self.ps
            plans.append((k, stay))
            need += self.pages(len(k)) - stay
        free = [p for p in range(self.np) if self.refs[p] == 0]
        if need > len(free):
            return False
        K, V, gone = self.K.copy(), self.V.copy(), []
        for i, (k, stay) in enumerate(plans):
            src_p, src_s = self.rows(i)
            n = self.pages(len(k)) - stay
            mine, free = free[:n], free[n:]
            gone += list(self.table[i, stay:self.pages(self.lens[i])])
            self.refs[mine] = 1
            self.table[i, stay:stay + n] = mine
            for j in range(stay * self.ps, len(k)):
                p, s = self.table[i, j // self.ps], j % self.ps
                self.K[p, s], self.V[p, s] = K[src_p[k[j]], src_s[k[j]]], V[src_p[k[j]], src_s[k[j]]]
            self.lens[i] = len(k)
        for p in gone:
            self.refs[p] -= 1
        return True

    def attend(self, q, cu, scale, causal):
        """(out, lse, weight, spread, every): per output weight = sum_t p_t |v_t| and every = sum_t |v_t|, per row spread =
        max_t scale sum_c |q_c k_tc|."""
        T, H, d = q.shape
        out, lse, every = np.zeros((T, H, d)), np.full((T, H), -np.inf), np.zeros((T, H, d))
        weight, spread = np.zeros((T, H, d)), np.zeros((T, H))
        for i in range(self.n):
            K, V = self.kv(i)
            nq, L = int(cu[i + 1] - cu[i]), len(K)
            for j in range(nq):
                sees = max(0, min(L, L - nq + j + 1)) if causal else L
                if not sees:
                    continue
                for h in range(H):
                    g = h // (H // K.shape[1])
                    x = q[cu[i] + j, h]
                    s = K[:sees, g] @ x * scale
                    m = s.max()
                    p = np.exp(s - m)
                    lse[cu[i] + j, h] = m + np.log(p.sum())
                    p /= p.sum()
                    out[cu[i] + j, h], weight[cu[i] + j, h] = p @ V[:sees, g], p @ np.abs(V[:sees, g])
                    every[cu[i] + j, h] = np.abs(V[:sees, g]).sum(0)
                    spread[cu[i] + j, h] = (np.abs(K[:sees, g]) @ np.abs(x)).max() * scale
        return out, lse, weight, spread, every
