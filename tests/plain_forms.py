"""Plain 64-bit forms of the attention over a paged cache, of the cache's bookkeeping and of the rules on logits, for the tests."""
import math

import torch


def half_step(dtype):
    """The most that one rounding to `dtype` is off, relative to the value."""
    return torch.finfo(dtype).eps / 2


def attend(k, v, table, q, n_queries, prefix, mask_bits=None, positions=None, window=0, sinks=0, scale=None, held_tokens=None):
    """k, v [n_pages, page, G, D], table [B, max_pages], q [B, N, H, D] on the CPU.  Returns out, lse and their tolerances, NaN for rows that
    are not written.

    The tolerance of out, with u the half step of the inputs' type: u |out| for the last rounding; of sum w |v| the share u (each weight is
    rounded to that type for the second product), keys * 2^-23 (its 32-bit sum), 2^-18 (exp2, the running maximum's factors, the division)
    and twice the error of a logit, which is an absolute error of scale * D * 2^-23 * sum |q k| from its 32-bit sum and of 2^-22 |logit| from
    its scaling.  The tolerance of lse is that error once and 2^-18 beside."""
    B, N, H, D = q.shape
    page, G = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    out = torch.full((B, N, H, D), math.nan, dtype=torch.float64)
    lse = torch.full((B, N, H), math.nan, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n, p = min(int(n_queries[b]), N), int(prefix[b])
        if n <= 0:
            continue
        keys = p + n if held_tokens is None else min(p + n, held_tokens[b])
        pages = table[b, :-(-keys // page)].long()
        kb = k[pages].reshape(-1, G, D)[:keys].double()
        vb = v[pages].reshape(-1, G, D)[:keys].double()
        see = torch.ones(n, keys, dtype=torch.bool)
        at = torch.arange(keys)
        own = p + torch.arange(n) if positions is None else positions[b, :n].long().clamp(min=p)
        for i in range(n):
            for j in range(keys - p):
                word = None if mask_bits is None else (int(mask_bits[b, i, j // 64]) if j < 64 * mask_bits.shape[2] else 0)
                see[i, p + j] = j <= i if mask_bits is None else bool(word >> (j % 64) & 1)
        if keys > p:
            at[p:] = own[:keys - p]
        if window:
            see &= (own[:, None] - at[None, :] < window) | (at < sinks)[None, :]
        for h in range(H):
            g = h // (H // G)
            kk = torch.where(see.any(0)[:, None], kb[:, g], 0.0)         # (what no row sees may hold anything)
            vv = torch.where(see.any(0)[:, None], vb[:, g], 0.0)
            qq = q[b, :n, h].double()
            x = (qq @ kk.T * scale).masked_fill(~see, -math.inf)
            top = x.amax(1, keepdim=True) if keys else torch.full((n, 1), -math.inf, dtype=torch.float64)
            w = torch.exp(x - torch.where(top > -math.inf, top, 0.0)).masked_fill(~see, 0.0)
            total = w.sum(1, keepdim=True)
            w = torch.where(total > 0, w / total, 0.0)
            finite = torch.where(torch.isfinite(vv), vv, 0.0)            # (a row that does not see a NaN does not get it)
            out[b, :n, h] = w @ finite
            lse[b, :n, h] = (top + total.log())[:, 0]
            away = (scale * D * 2.0 ** -23 * (qq.abs() @ kk.abs().nan_to_num(0.0).T) + 2.0 ** -22 * x.abs().nan_to_num(0.0, 0.0, 0.0))
            away = torch.where(see, away, 0.0).amax(1, keepdim=True) if keys else torch.zeros(n, 1)
            u = half_step(q.dtype)
            tol[b, :n, h] = u * out[b, :n, h].abs() + (u + keys * 2.0 ** -23 + 2.0 ** -18 + 2.1 * away) * (w @ finite.abs())
            tol_lse[b, :n, h] = away[:, 0] + 2.0 ** -18
    return out, lse, tol, tol_lse


class Pages:
    """The cache's bookkeeping, slot by slot."""

    def __init__(self, table, held, refs, page):
        self.table, self.held, self.refs, self.page = table.clone(), held.clone(), refs.clone(), page
        self.status = [0] * len(held)

    def _free(self):
        return [i for i, r in enumerate(self.refs.tolist()) if r == 0]

    def reserve(self, length):
        free, at, short = self._free(), 0, False
        for b, n in enumerate(length):
            if n < 0 or n > self.table.shape[1] * self.page:
                self.status[b] |= 64
                continue
            need = -(-n // self.page) - int(self.held[b])
            if need <= 0:
                continue
            short = short or at + need > len(free)
            if short:
                self.status[b] |= 32
                continue
            for page in free[at:at + need]:
                self.table[b, self.held[b]] = page
                self.refs[page] = 1
                self.held[b] += 1
            at += need

    def release(self, keep):
        for b, n in enumerate(keep):
            if n < 0:
                self.status[b] |= 64
                continue
            while self.held[b] > -(-n // self.page):
                self.held[b] -= 1
                self.refs[self.table[b, self.held[b]]] -= 1
                self.table[b, self.held[b]] = -1

    def fork(self, source, length):
        """Returns the slots that were made and the (old page, new page, tokens) that were copied."""
        free, held, copies, made, short = self._free(), self.held.tolist(), [], [0] * len(source), False
        for b, (s, n) in enumerate(zip(source, length)):
            if s < 0:
                continue
            if s >= len(source) or s == b or source[s] >= 0 or held[b] or n < 0 or n > held[s] * self.page:
                self.status[b] |= 64
                continue
            full, rest = divmod(n, self.page)
            if rest and (short or len(copies) == len(free)):
                short = True
                self.status[b] |= 32
                continue
            made[b] = 1
            self.table[b, :full] = self.table[s, :full]
            for page in self.table[s, :full].tolist():
                self.refs[page] += 1
            if rest:
                new = free[len(copies)]
                copies.append((int(self.table[s, full]), new, rest))
                self.table[b, full], self.refs[new] = new, 1
            self.held[b] = full + (rest > 0)
        return made, copies


def penalize(logits, n_rows=None, counts=None, repetition=None, frequency=None, presence=None, bias=None, allowed=None,
             node_token=None, node_parent=None, row_node=None):
    """logits [B, R, V] on the CPU -> 64-bit rows, NaN where nothing is written; and which of them a row's text has."""
    B, R, V = logits.shape
    out = torch.full((B, R, V), math.nan, dtype=torch.float64)
    touched = torch.zeros(B, R, V, dtype=torch.bool)
    for b in range(B):
        for r in range(R if n_rows is None else min(int(n_rows[b]), R)):
            c = torch.zeros(V, dtype=torch.float64) if counts is None else counts[b].double()
            if node_token is not None:
                node, left = (r if row_node is None else int(row_node[b, r])), 33
                while 0 <= node < node_token.shape[1] and left:
                    t = int(node_token[b, node])
                    if 0 <= t < V:
                        c[t] += 1
                    node, left = int(node_parent[b, node]), left - 1
            x = logits[b, r].double()
            rep = 1.0 if repetition is None else float(repetition[b])
            freq = 0.0 if frequency is None else float(frequency[b])
            pres = 0.0 if presence is None else float(presence[b])
            x = torch.where(c > 0, torch.where(x > 0, x / rep, x * rep) - freq * c - pres, x)
            if bias is not None:
                x = x + (bias if bias.dim() == 1 else bias[b]).double()
            if allowed is not None:
                words = allowed[b] if allowed.dim() == 2 else allowed[b, r]
                on = (words.long()[torch.arange(V) // 32] >> (torch.arange(V) % 32)) & 1
                x = torch.where(on > 0, x, -math.inf)
            out[b, r], touched[b, r] = x, c > 0
    return out, touched
