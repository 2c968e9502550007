"""The definition of attention to a paged cache in 64 bits, with torch on the tensors' device: past_ref.paged for calls that are too large for it."""
import math

import torch


def paged(q, k_pages, v_pages, table, page, q_len, own_len, table_row, prefix=None, prefix_len=(), prefix_table_row=(), causal=True, scale=None):
    """What past_ref.paged gives, as numpy arrays.  Values that a query sees are finite."""
    _, heads, d = q.shape
    n_pages, kv = k_pages.shape[:2]
    group, scale = heads // kv, scale or 1 / math.sqrt(d)

    def rows_of(table_row, length):
        """Keys and values [kv, rows, d] of the rows that there are, and their numbers."""
        j = torch.arange(length, device=q.device)
        pages = table[table_row].long()[j // page]
        there = (pages >= 0) & (pages < n_pages)
        j, pages = j[there], pages[there]
        return [t[pages, :, j % page].double().transpose(0, 1).contiguous() for t in (k_pages, v_pages)] + [j]

    prefixes = {g: rows_of(prefix_table_row[g], prefix_len[g]) for g in {p for p in prefix or () if p >= 0}}
    out, mass = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    lse, size = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    at = 0
    for i, (n, m) in enumerate(zip(q_len, own_len)):
        k, v, j = rows_of(table_row[i], m)
        sees = (j <= m - n + torch.arange(n, device=q.device)[:, None]) | (not causal)
        of = -1 if prefix is None else prefix[i]
        if of >= 0:
            pre_k, pre_v, pre_j = prefixes[of]
            k, v, sees = torch.cat([pre_k, k], 1), torch.cat([pre_v, v], 1), torch.cat([torch.ones(n, len(pre_j), dtype=torch.bool, device=q.device), sees], 1)
        # (a key that nobody sees may hold anything)
        used = sees.any(0)
        k, v, sees = k[:, used], v[:, used], sees[:, used]
        if n and k.shape[1]:
            qq = q[at: at + n].double().view(n, kv, group, d).permute(1, 0, 2, 3).reshape(kv, n * group, d)
            hidden = ~sees.repeat_interleave(group, 0)
            score = (scale * (qq @ k.transpose(1, 2).contiguous())).masked_fill(hidden, -math.inf)
            top = score.amax(2, keepdim=True)
            e = torch.exp(score - torch.where(top == -math.inf, 0, top))
            total = e.sum(2, keepdim=True)
            w = e / torch.where(total == 0, 1, total)
            back = lambda x: x.view(kv, n, group, -1).permute(1, 0, 2, 3).reshape(n, heads, -1)       # noqa: E731
            out[at: at + n], mass[at: at + n] = back(w @ v), back(w @ v.abs())
            lse[at: at + n] = back(top + total.log())[:, :, 0]
            size[at: at + n] = back((scale * (qq.abs() @ k.abs().transpose(1, 2).contiguous())).masked_fill(hidden, 0).amax(2, keepdim=True))[:, :, 0]
        at += n
    return [x.cpu().numpy() for x in (out, lse, mass, size)]
