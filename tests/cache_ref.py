"""Plain 64-bit (or bit by bit, where the library's recipe is one of float32 roundings) forms of the serving calls between the
projections, for the tests: rotations, the 8-bit cache and its pages, attention."""
import math

import numpy as np

F = np.float32


def rotate(x, positions, freq, interleaved, norm, gain, eps, offset, amplitude):
    """float64 [n][heads][d] of x (numpy)."""
    y = x.astype(np.float64)
    d = y.shape[2]
    if norm:
        y = y / np.sqrt((y * y).mean(2, keepdims=True) + eps)
        if gain is not None:
            y = y * (offset + gain.astype(np.float64))
    out = y.copy()
    half = len(freq)
    for i in range(half):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        w = positions.astype(np.float64) * freq[i]
        c, s = np.cos(w)[:, None], np.sin(w)[:, None]
        out[:, :, p] = amplitude * (y[:, :, p] * c - y[:, :, q] * s)
        out[:, :, q] = amplitude * (y[:, :, p] * s + y[:, :, q] * c)
    return out, y


class Pool:
    """A cache as lists and numpy arrays: codes [pages][heads][block][d] of both sides, rows of pages."""

    def __init__(self, sequences, pages, heads, d, block, width):
        self.block, self.width, self.pages = block, width, pages
        self.codes = [np.zeros((pages, heads, block, d), np.int8) for _ in range(2)]
        self.scales = [np.zeros((pages, heads), F) for _ in range(2)]
        self.table = -np.ones((sequences, width), np.int32)
        self.lengths = np.zeros(sequences, np.int32)
        self.refs = np.zeros(pages, np.int32)

    def blocks(self, tokens):
        return -(-int(tokens) // self.block)

    def reserve(self, counts):
        """The new tokens' positions, or how many pages lack."""
        want, over = [], 0
        for i, n in enumerate(counts):
            have, need = self.blocks(self.lengths[i]), self.blocks(self.lengths[i] + n)
            over += max(0, need - self.width)
            last = self.table[i, have - 1] if have else -1
            copy = bool(n > 0 and self.lengths[i] % self.block and 0 <= last < self.pages and self.refs[last] > 1)
            want.append((copy, last, have, min(need, self.width) - have))
        total = sum(c + m for c, _, _, m in want)
        free = np.flatnonzero(self.refs == 0)
        if over or len(free) < total:
            return None, over or total - len(free)
        free, positions = list(free[:total]), []
        for i, (copy, last, have, more) in enumerate(want):
            if copy:
                p = free.pop(0)
                for side in range(2):
                    self.codes[side][p] = self.codes[side][last]
                    self.scales[side][p] = self.scales[side][last]
                self.refs[last] -= 1
                self.refs[p] = 1
                self.table[i, have - 1] = p
            for b in range(more):
                p = free.pop(0)
                self.refs[p] = 1
                self.table[i, have + b] = p
            positions += list(range(self.lengths[i], self.lengths[i] + counts[i]))
            self.lengths[i] += counts[i]
        return np.array(positions, np.int32), 0

    def reorder(self, sources):
        table, lengths = self.table.copy(), self.lengths.copy()
        for i, s in enumerate(sources):
            if s == i:
                continue
            some = 0 <= s < len(lengths)
            self.lengths[i] = lengths[s] if some else 0
            self.table[i] = -1
            if some:
                b = self.blocks(lengths[s])
                self.table[i, :b] = table[s, :b]
        self.refs = np.bincount(self.table[self.table >= 0], minlength=self.pages).astype(np.int32)

    def compact(self):
        used = self.refs > 0
        count = int(used.sum())
        src, dst = np.flatnonzero(used[count:]) + count, np.flatnonzero(~used[:count])
        to = np.arange(self.pages)
        to[src] = dst
        for side in range(2):
            self.codes[side][dst] = self.codes[side][src]
            self.scales[side][dst] = self.scales[side][src]
        self.refs[dst] = self.refs[src]
        self.refs[src] = 0
        self.table = np.where(self.table >= 0, to[np.maximum(self.table, 0)], self.table).astype(np.int32)
        return count

    def append(self, k, v, starts, longest=None):
        """The recipe of float32 roundings, bit by bit."""
        B = self.block
        with np.errstate(all="ignore"):
            for i in range(len(self.lengths)):
                n = starts[i + 1] - starts[i]
                length = min(int(self.lengths[i]), self.width * B)
                pos0 = length - n
                last = min(length, pos0 + (n if longest is None else longest))
                for b in range(max(pos0, 0) // B, self.blocks(last) if last > 0 else 0):
                    first, end = max(pos0, b * B), min(last, (b + 1) * B)
                    if first < 0:
                        first = 0
                    page = self.table[i, b]
                    if first >= end or not 0 <= page < self.pages:
                        continue
                    f = first - b * B
                    for side, x in enumerate((k, v)):
                        new = x[starts[i] + first - pos0:starts[i] + end - pos0].astype(F)        # [tokens][heads][d]
                        for h in range(new.shape[1]):
                            self._store(self.codes[side][page, h], self.scales[side], (page, h), new[:, h], f)

    @staticmethod
    def _store(codes, scales, at, new, f):
        def mag(x):
            return np.abs(np.asarray(x, F)).view(np.uint32)

        old = np.abs(F(scales[at])) if f > 0 else F(0)
        top = mag(new).max().astype(np.uint32).view(F) / F(127)
        s = max(mag(old)[()], mag(top)[()])
        s = np.uint32(s).view(F)
        number = np.isfinite(s)
        if f > 0 and mag(s)[()] != mag(old)[()]:
            ratio = F(old / s) if number else F(0)
            codes[:f] = np.rint(codes[:f].astype(F) * ratio).astype(np.int8)
        inv = min(F(1) / s, np.finfo(F).max) if number and s > 0 else F(0)
        q = np.clip(np.rint((new * F(inv)).astype(F)), -127, 127) if number else np.zeros_like(new)
        codes[f:f + len(new)] = q.astype(np.int8)
        scales[at] = s

    def values(self, side, i, begin, n):
        """float32 [n][heads][d]; positions and pages that are not there give zeros."""
        out = np.zeros((n,) + self.codes[side].shape[1:2] + self.codes[side].shape[3:], F)
        length = min(int(self.lengths[i]), self.width * self.block)
        for j in range(n):
            p = begin + j
            if 0 <= p < length:
                page = self.table[i, p // self.block]
                if 0 <= page < self.pages:
                    out[j] = self.codes[side][page, :, p % self.block].astype(F) * self.scales[side][page][:, None]
        return out


def attend(torch, cache, q, starts, scale, softcap, window, causal):
    """float64 (out, lse, weight, size, floor) on q's device from a library cache: weight = sum_t p |V| (what errors of the weights are counted
    in), size [n][heads_q] = the largest scale * sum_c |q K| over a row's keys (what errors of the scores are counted in), floor = sum_t |c| over a
    row's keys times their largest scale of v, c the codes (what weights too small for float16's 11 bits are counted in)."""
    n, hq, d = q.shape
    pages, heads, B, _ = cache.k.shape
    dev = q.device
    out = torch.full((n, hq, d), float("nan"), dtype=torch.float64, device=dev)
    weight, floor, lse = torch.zeros_like(out), torch.zeros_like(out), torch.full((n, hq), float("nan"), dtype=torch.float64, device=dev)
    size = torch.zeros_like(lse)
    width = cache.table.shape[1]
    for i in range(len(starts) - 1):
        lo, hi = starts[i], starts[i + 1]
        if hi <= lo:
            continue
        length = min(int(cache.lengths[i]), width * B)
        pos = torch.arange(length - (hi - lo), length, device=dev)[:, None]
        page = cache.table[i, :-(-length // B)].long()
        there = ((page >= 0) & (page < pages)).repeat_interleave(B)[:length]
        page = page.clamp(0, pages - 1)
        key = torch.arange(length, device=dev)[None, :]
        live = there[None, :].expand(hi - lo, -1).clone()
        if causal:
            live &= key <= pos
        if window:
            live &= key > pos - window
        for h in range(heads):
            K = (cache.k[page, h].double() * cache.kscale[page, h].double()[:, None, None]).reshape(-1, d)[:length]
            V = (cache.v[page, h].double().transpose(1, 2) * cache.vscale[page, h].double()[:, None, None]).reshape(-1, d)[:length]
            used = live.any(0)
            codes = cache.v[page, h].double().transpose(1, 2).reshape(-1, d)[:length].abs()
            vs = torch.where(live, cache.vscale[page, h].double().repeat_interleave(B)[None, :length], torch.zeros((), dtype=torch.float64, device=dev))
            most = (live.double() @ codes) * (vs.amax(1, keepdim=True) if length else 0.0)
            K = torch.where(used[:, None], K, torch.zeros_like(K))
            V = torch.where(used[:, None], V, torch.zeros_like(V))
            for g in range(h * (hq // heads), (h + 1) * (hq // heads)):
                x = q[lo:hi, g].double()
                s = x @ K.t() * scale
                size[lo:hi, g] = torch.where(live, (x.abs() @ K.abs().t()) * abs(scale), torch.zeros_like(s)).amax(1) if length else 0.0
                if softcap:
                    s = softcap * torch.tanh(s / softcap)
                s = torch.where(live, s, torch.full_like(s, -math.inf))
                norm = torch.logsumexp(s, 1) if length else torch.full((hi - lo,), -math.inf, dtype=torch.float64, device=dev)
                p = torch.where(live, torch.exp(s - torch.where(live.any(1), norm, torch.zeros_like(norm))[:, None]), torch.zeros_like(s))
                out[lo:hi, g] = p @ V
                weight[lo:hi, g] = p @ V.abs()
                lse[lo:hi, g] = norm
                floor[lo:hi, g] = most
    return out, lse, weight, size, floor
