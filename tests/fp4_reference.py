"""Plain implementations of the cache in 4 bits and of the reordering of beams: numpy and Python loops, written from their contracts."""
import numpy as np
import torch

from tests import tree_reference as R


def small_floats(exponents, fractions, bias):
    """What a small float can be, ascending: its bits are the place."""
    return np.array([m / fractions * 2.0 ** (1 - bias) if e == 0 else (1 + m / fractions) * 2.0 ** (e - bias) for e in range(exponents) for m in range(fractions)])


E2M1 = small_floats(4, 2, 1)
E4M3 = small_floats(16, 8, 7)[:127]                            # (the last bits are NaN)


def nearest(x, values):
    """Places of the nearest of the ascending values, halfway the even place, beyond the last the last."""
    hi = np.minimum(np.searchsorted(values, x), len(values) - 1)
    lo = np.maximum(hi - 1, 0)
    below, above = x - values[lo], values[hi] - x
    return np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def quantise(x, unit=None):
    """(codes [..., D / 2], scales [..., D / 16] as bytes) of x [..., D] (a torch tensor): the contract's two quotients in fp32, everything else by distance in 64 bits."""
    x = x.float().numpy()
    with np.errstate(all="ignore"):
        if unit is not None:
            x = x / np.float32(unit)
        x = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
        nan = np.isnan(x).any(-1)
        top = np.abs(x).max(-1)
        scale = nearest((top / np.float32(6)).astype(np.float64), E4M3)
        s = E4M3[scale][..., None]
        number = nearest(np.where(s > 0, np.abs(x) / s.astype(np.float32), 0).astype(np.float64), E2M1) + 8 * np.signbit(x)
    scale = np.where(nan, 127, scale)
    number = number.reshape(*number.shape[:-2], number.shape[-2] * 16)
    return torch.from_numpy((number[..., ::2] | number[..., 1::2] << 4).astype(np.uint8)), torch.from_numpy(scale.astype(np.uint8))


def values(codes, scales):
    """float64 values of codes and scales."""
    c, s = codes.numpy(), np.append(E4M3, np.nan)[scales.numpy() & 127]
    number = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], c.shape[-1] * 2)
    v = np.where(number >= 8, -1.0, 1.0) * E2M1[number & 7]
    return torch.from_numpy(v * np.repeat(s, 16, -1))


class Pages(R.Pages):
    """... with beams.  For a cache in 4 bits kv holds a token and head's bytes, codes and scales together."""

    def reorder(self, groups, parents):
        """Returns the status bits; too few pages: nothing changes."""
        before = [(list(t), n) for t, n in zip(self.table, self.length)]
        refs, status, plan = list(self.refs), 0, []
        known = lambda s: 0 <= s < len(before)  # noqa: E731
        for seqs, up in zip(groups, parents):
            own = []
            for i, (s, p) in enumerate(zip(seqs, up)):
                if not known(s):
                    status |= 4
                    own.append(None)
                elif p != -1 and not (0 <= p < len(seqs) and known(seqs[p])):
                    status |= 4
                    own.append(i)
                else:
                    own.append(p)
            for i, (s, p) in enumerate(zip(seqs, own)):
                if p is None:
                    continue
                for page in before[s][0]:
                    refs[page] -= 1
                if p == -1:
                    plan.append((s, [], 0, None))
                    continue
                table, n = before[seqs[p]]
                children = [j for j in range(len(seqs)) if own[j] == p]
                heir = p if p in children else children[0]
                full, part = n // self.page, n % self.page
                keep = table[:full + (part > 0 and i == heir)]
                for page in keep:
                    refs[page] += 1
                plan.append((s, keep, n, table[full] if part and i != heir else None))
        free = [p for p, n in enumerate(refs) if n == 0]
        if sum(x[3] is not None for x in plan) > len(free):
            return status | 1
        content = self.kv.clone()
        for s, keep, n, copied in plan:
            self.table[s], self.length[s] = list(keep), n
            if copied is not None:
                p = free.pop(0)
                refs[p] = 1
                self.kv[:, :, p, :n % self.page] = content[:, :, copied, :n % self.page]
                self.table[s].append(p)
        self.refs = refs
        return status
