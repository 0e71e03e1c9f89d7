"""Plain references of the 4-bit matrices and the 4-bit sequence cache, in 64 bits (numpy and torch on the CPU or GPU), sharing no code with the library."""
import math

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantise(x):
    """x [..., cols] -> values that its 4-bit form stands for (float64), codes [..., cols] (0..15), scale bytes [..., cols / 32]."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    finite = torch.isfinite(b).all(-1)
    safe = torch.where(finite & (top > 0), top, torch.ones_like(top))
    e = (torch.frexp(safe).exponent - 1 - 2).clamp(min=-127)
    e = torch.where(finite & (top > 0), e, torch.full_like(e, -127))
    y = torch.ldexp(b.abs(), -e.unsqueeze(-1))
    y = torch.where(torch.isfinite(y), y, torch.zeros_like(y))
    grid = GRID.to(x.device)
    code = torch.zeros_like(y, dtype=torch.int64)
    for i in range(1, 8):   # midpoint between two neighbours: to the even code
        mid = (grid[i - 1] + grid[i]) / 2
        code = torch.where((y > mid) | ((y == mid) & (i % 2 == 0)), torch.full_like(code, i), code)
    v = torch.copysign(torch.ldexp(grid[code], e.unsqueeze(-1)), b)
    v = torch.where(finite.unsqueeze(-1), v, torch.full_like(v, math.nan))
    byte = torch.where(finite, e + 127, torch.full_like(e, 255))
    code = torch.where(torch.signbit(b), code + 8, code)
    code = torch.where(finite.unsqueeze(-1), code, torch.zeros_like(code))
    return v.flatten(-2), code.flatten(-2).to(torch.uint8), byte.to(torch.uint8)


def stored_values(codes, scales):
    """Packed codes [..., w / 2] and scale bytes [..., w / 32] -> float64 values."""
    grid = torch.cat((GRID, -GRID)).to(codes.device)
    v = grid[torch.stack((codes & 15, codes >> 4), -1).long()].flatten(-2).unflatten(-1, (-1, 32))
    s = torch.where(scales == 255, torch.full(scales.shape, math.nan, dtype=torch.float64, device=scales.device),
                    torch.ldexp(torch.ones(scales.shape, dtype=torch.float64, device=scales.device), scales.int() - 127))
    return (v * s.unsqueeze(-1)).flatten(-2)


def scale_places(rows, blocks):
    """Index of byte (row, block) in the tiled buffer of a matrix's scales."""
    tiles = -(-blocks // 4)
    r, b = torch.arange(rows).unsqueeze(1), torch.arange(blocks).unsqueeze(0)
    return ((r // 128) * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def attention(q, k, v, scale):
    """q [rows, d], k, v [keys, d] in float64: softmax(scale q k^T) v, and what its error bounds need: the rows' sums of w |v - out|, of w |v| and
    (smallest weights a kernel can tell from nothing) of |v|, and the largest sum of |q k| scale with the product of the largest elements added."""
    if k.shape[0] == 0:
        z = torch.zeros(q.shape[0], v.shape[1], dtype=torch.float64, device=q.device)
        return z, z, (z, z), 0.0
    s = q @ k.T * scale
    w = torch.exp(s - s.amax(1, keepdim=True))
    w = w / w.sum(1, keepdim=True)
    out = w @ v
    spread = torch.stack([(w[i].unsqueeze(1) * (v - out[i]).abs()).sum(0) for i in range(q.shape[0])])
    return out, spread, (w @ v.abs(), v.abs().sum(0).expand_as(out)), float(((q.abs() @ k.abs().T).max() + q.abs().max() * k.abs().max()) * scale)


def attention_bound(dtype, out, spread, mass, reach, d):
    """Largest error of an output: scores are sums of d fp32 products (each sum off by at most d 2^-24 of the products' magnitudes), the exponential by
    2^-21; weights are fp32 or rounded to bf16 (half a step: 2^-8) or fp16 (2^-11); the output is rounded once to its type.
    fp16 weights are between 2^7 and 2^15 at their largest and have steps of 2^-24 at their smallest, so each is off by up to 2^-25 / 2^7 of the largest
    weight (at most 1) too.  Queries and keys held in fp16 relative to their largest elements are off by up to 2^-25 of those per element, a score by d 2^-24 of
    the product of the largest."""
    mass, total = mass
    weight = 2 * (d * 2.0 ** -24 * reach + 2.0 ** -20)
    if dtype == torch.bfloat16:
        return (weight + 1.01 * 2.0 ** -8) * spread + 2.0 ** -11 * mass + 2.0 ** -31 * total + 1.01 * 2.0 ** -8 * out.abs() + 1e-37
    return (weight + 2.0 ** -20) * mass + 2.0 ** -23 * out.abs() + 1e-37


class Books:
    """The cache's books as Python lists: what every call has to leave behind."""

    def __init__(self, n_pages, page_rows, n_seqs, max_pages):
        self.R, self.max_pages, self.n_seqs = page_rows, max_pages, n_seqs
        self.pages = [[] for _ in range(n_seqs)]
        self.length = [0] * n_seqs
        self.refs = [0] * n_pages
        self.free = list(range(n_pages))[::-1]
        self.rows = [[] for _ in range(n_seqs)]   # tags of the rows, to compare contents with
        self.bad = self.full = False

    def _standing(self, ids):
        seen, out = set(), []
        for i, s in enumerate(ids):
            ok = 0 <= s < self.n_seqs and s not in seen
            if 0 <= s < self.n_seqs:
                seen.add(s)
            if not ok:
                self.bad = True
            out.append(ok)
        return out

    def _release(self, entries):
        """entries: (position, sequence).  References first, then the pages that nobody has, last entry's last page first."""
        for _, s in entries:
            for p in self.pages[s]:
                self.refs[p] -= 1
        keys = {}
        for i, s in entries:
            for x, p in enumerate(self.pages[s]):
                if self.refs[p] == 0:
                    keys[p] = min(keys.get(p, (i, x)), (i, x))
        self.free += [p for p, _ in sorted(keys.items(), key=lambda kv: kv[1], reverse=True)]
        for _, s in entries:
            self.pages[s], self.length[s], self.rows[s] = [], 0, []

    def free_seqs(self, ids):
        self._release([(i, s) for i, (s, ok) in enumerate(zip(ids, self._standing(ids))) if ok])

    def share(self, src, dst, copy):
        ok = self._standing(dst)
        listed = {s for s in dst if 0 <= s < self.n_seqs}
        for i, s in enumerate(src):
            if ok[i] and not (0 <= s < self.n_seqs and s not in listed):
                ok[i], self.bad = False, True
        entries = [(i, dst[i]) for i in range(len(dst)) if ok[i]]
        self._release(entries)
        available, spent = len(self.free), 0
        for i, s in entries:
            f = src[i]
            if not copy:
                self.pages[s] = list(self.pages[f])
                for p in self.pages[s]:
                    self.refs[p] += 1
            else:
                need = len(self.pages[f])
                spent += need
                if need and spent > available:
                    self.full = True
                    continue
                self.pages[s] = [self.free.pop() for _ in range(need)]
                for p in self.pages[s]:
                    self.refs[p] = 1
            self.length[s], self.rows[s] = self.length[f], list(self.rows[f])

    def append(self, ids, counts, tags):
        ok = self._standing(ids)
        shared_at_start = {}
        for i, s in enumerate(ids):
            if ok[i]:
                shared_at_start[i] = bool(counts[i]) and self.length[s] % self.R > 0 and self.refs[self.pages[s][-1]] > 1
        available, spent, given_up, at = len(self.free), 0, {}, 0
        for i, s in enumerate(ids):
            mine, at = tags[at:at + counts[i]], at + counts[i]
            if not ok[i]:
                continue
            if self.length[s] + counts[i] > self.max_pages * self.R:
                self.full = True
                continue
            need = -(-(self.length[s] + counts[i]) // self.R) - len(self.pages[s]) + shared_at_start[i]
            spent += need
            if need and spent > available:
                self.full = True
                continue
            if shared_at_start[i]:
                old = self.pages[s][-1]
                self.refs[old] -= 1
                given_up.setdefault(old, i)
                self.pages[s][-1] = self.free.pop()
                self.refs[self.pages[s][-1]] = 1
                need -= 1
            for _ in range(need):
                self.pages[s].append(self.free.pop())
                self.refs[self.pages[s][-1]] = 1
            self.length[s] += counts[i]
            self.rows[s] += mine
        self.free += [p for p, _ in sorted(given_up.items(), key=lambda kv: kv[1], reverse=True) if self.refs[p] == 0]

    def compact(self, n_pages):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        out = Books(n_pages, self.R, self.n_seqs, self.max_pages)
        if len(live) > n_pages:
            out.full = True
            return out
        place = {p: i for i, p in enumerate(live)}
        out.pages = [[place[p] for p in ps] for ps in self.pages]
        out.length, out.rows = list(self.length), [list(r) for r in self.rows]
        out.refs = [self.refs[p] for p in live] + [0] * (n_pages - len(live))
        out.free = list(range(len(live), n_pages))[::-1]
        return out
