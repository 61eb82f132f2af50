"""Independent 64-bit oracle of what surrounds the products and attention of a step: placing and trimming (sequence by sequence, page by
page, from the text of include/lutgemm.h), the norm, low-rank adapters.  Test infrastructure."""
import numpy as np


# ---- where tokens stand ----------------------------------------------------------------------------
class Pages:
    def __init__(self, pages, page_tokens, seqs, table_pages):
        self.pages, self.page_tokens, self.table_pages = pages, page_tokens, table_pages
        self.free = list(range(pages - 1, -1, -1))            # the last is taken next
        self.table = [[] for _ in range(seqs)]

    def place(self, past, fresh, tokens, most):
        first, positions, owner, slots = [0], [], [], []
        waiting = False
        for s, mine in enumerate(self.table):
            n = int(fresh[s])
            end = int(past[s]) + n
            if not waiting and 0 < n <= most and past[s] >= 0 and end <= self.table_pages * self.page_tokens:
                need = max(0, -(-end // self.page_tokens) - len(mine))
                if len(positions) + n > tokens or need > len(self.free):
                    waiting = True
                else:
                    for _ in range(need):
                        mine.append(self.free.pop())
                    for p in range(int(past[s]), end):
                        positions.append(p)
                        owner.append(s)
                        slots.append(mine[p // self.page_tokens] * self.page_tokens + p % self.page_tokens)
            first.append(len(positions))
        rest = tokens - len(positions)
        return (np.array(first, np.int32), np.array(positions + [0] * rest, np.int32), np.array(owner + [-1] * rest, np.int32),
                np.array(slots + [-1] * rest, np.int64))

    def trim(self, lengths):
        back = []
        for s, mine in enumerate(self.table):
            if lengths[s] >= 0:
                keep = min(-(-int(lengths[s]) // self.page_tokens), len(mine))
                back += mine[keep:]
                del mine[keep:]
        self.free += back[::-1]

    def arrays(self):
        table = np.full((len(self.table), self.table_pages), -1, np.int32)
        for s, mine in enumerate(self.table):
            table[s, :len(mine)] = mine
        return np.array(self.free, np.int32), np.array([len(t) for t in self.table], np.int32), table


# ---- norm ------------------------------------------------------------------------------------------
def rms_norm(x, residual, weight, eps):
    """x [tokens][n]; returns s and y in 64 bits."""
    s = x.astype(np.float64) + (0.0 if residual is None else residual.astype(np.float64))
    with np.errstate(invalid="ignore", over="ignore"):
        y = s / np.sqrt((s * s).mean(1, keepdims=True) + eps)
        return s, y if weight is None else y * weight.astype(np.float64)


# ---- adapters --------------------------------------------------------------------------------------
def adapt(x, base, down, up, ranks, scales, of):
    """of: the adapter of every token (or none, out of range).  Returns y and what error bounds need: sum over ranks and columns of
    |c B| |A| |x|, and of |c B| |h|."""
    y = base.astype(np.float64)
    reach, mass = np.zeros_like(y), np.zeros_like(y)
    for t, a in enumerate(of):
        if not 0 <= a < len(down):
            continue
        r = down.shape[1] if ranks is None else int(ranks[a])
        c = 1.0 if scales is None else float(scales[a])
        A, B, v = down[a, :r].astype(np.float64), up[a, :, :r].astype(np.float64), x[t].astype(np.float64)
        h = A @ v
        y[t] += c * (B @ h)
        reach[t] = abs(c) * (np.abs(B) @ (np.abs(A) @ np.abs(v)))
        mass[t] = abs(c) * (np.abs(B) @ np.full(r, np.abs(h).max() if r else 0.0))
    return y, reach, mass
