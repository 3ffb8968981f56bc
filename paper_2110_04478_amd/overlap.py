"""Whether strided views of memory have a byte in common, from addresses and strides alone.

A view is (address, levels, element bytes): its elements begin at address + the sum of k_i * stride_i
over its levels (stride in bytes, most), 0 <= k_i <= most.  Two views share a byte where a sum of
bounded multiples takes one value; `_reaches` decides that exactly.  Before it comes what settles
nearly everything: views whose spans are apart, and views that are apart modulo one of their
strides (columns of one matrix, every other element)."""
from __future__ import annotations

import bisect

_STEPS = 1 << 20   # of the exact search in one question, a second or two; beyond them the answer is "shared"
_PAIR = 8          # steps that a pair of views costs at least
_MODULI = 8


class _Undecided(Exception):
    pass


def view_of(t) -> tuple:
    size = t.element_size()
    if t.is_contiguous():
        return t.data_ptr(), [(size, t.numel() - 1)], size
    return t.data_ptr(), [(s * size, n - 1) for n, s in zip(t.shape, t.stride()) if n != 1 and s], size


def _reaches(levels, at, steps) -> bool:
    """Whether sum of k_i * stride_i == at for some 0 <= k_i <= most_i.  steps: [what is left]."""
    merged = {}
    for s, n in levels:
        if n:
            merged[s] = merged.get(s, 0) + n
    levels = sorted(merged.items())
    reach, whole = [0], [True]   # of the levels below; whether these give every sum up to it
    for s, n in levels:
        whole.append(whole[-1] and s <= reach[-1] + 1)
        reach.append(reach[-1] + s * n)
    seen = set()

    def search(k, at):   # the levels below k
        if at < 0 or at > reach[k]:
            return False
        if whole[k]:
            return True
        if (k, at) in seen:
            return False
        s, n = levels[k - 1]
        for x in range(max(0, -((reach[k - 1] - at) // s)), min(n, at // s) + 1):
            steps[0] -= 1
            if steps[0] < 0:
                raise _Undecided
            if search(k - 1, at - x * s):
                return True
        seen.add((k, at))
        return False

    return search(len(levels), at)


def _two_share(a, b, steps) -> bool:
    # address_a + sums_a + byte_a == address_b + sums_b + byte_b, with b's multiples counted from the other end
    turned = sum(s * n for s, n in b[1]) + b[2] - 1
    steps[0] -= _PAIR
    return _reaches([*a[1], *b[1], (1, a[2] + b[2] - 2)], b[0] - a[0] + turned, steps)


def repeats(t) -> bool:
    """Whether two elements of a tensor are one place in memory."""
    if t.is_contiguous() or t.numel() < 2:
        return False
    levels = sorted((s, n - 1) for n, s in zip(t.shape, t.stride()) if n != 1)
    if levels[0][0] == 0:
        return True
    reach = 0
    for s, n in levels:
        if s <= reach:
            break
        reach += s * n
    else:
        return False   # every step is longer than all shorter ones together
    # A difference of two places that is none: its longest step that counts k >= 1 times, others -n .. n.
    try:
        steps = [_STEPS]
        for i, (s, n) in enumerate(levels):
            below = levels[:i]
            if _reaches([(s, n - 1)] + [(x, 2 * m) for x, m in below], sum(x * m for x, m in below) - s, steps):
                return True
        return False
    except _Undecided:
        return True


def _groups(spans):
    """Numbers of the views whose spans (begin, end, number) hang together, two at least."""
    spans.sort()
    group, reach = [], -1
    for begin, end, i in spans:
        if begin >= reach:
            if len(group) > 1:
                yield group
            group = [i]
            reach = end
        else:
            group.append(i)
            if end > reach:
                reach = end
    if len(group) > 1:
        yield group


def _share(views, group, moduli, steps) -> bool:
    group = sorted(set(group))
    if len(group) < 2 or not any(views[i][3] for i in group):
        return False
    if moduli is None:   # strides of many of them, then long ones, first
        count = {}
        for i in group:
            for s, _ in views[i][1]:
                count[s] = count.get(s, 0) + 1
        moduli = sorted(count, key=lambda s: (-count[s], -s))[:_MODULI]
    if moduli:
        m, spans = moduli[0], []
        for i in group:
            at, levels, size, _ = views[i]
            begin, length = at % m, sum(s * n for s, n in levels if s % m) + size
            if length >= m:
                spans.append((0, m, i))
            else:
                spans.append((begin, min(begin + length, m), i))
                if begin + length > m:
                    spans.append((0, begin + length - m, i))
        return any(_share(views, g, moduli[1:], steps) for g in _groups(spans))
    group.sort(key=lambda i: views[i][0])
    targets = [k for k, i in enumerate(group) if views[i][3]]
    for k, i in enumerate(group):
        at, levels, size, written = views[i]
        end = at + sum(s * n for s, n in levels) + size
        for j in range(k + 1, len(group)) if written else targets[bisect.bisect(targets, k):]:
            if views[group[j]][0] >= end:
                break
            if _two_share(views[i], views[group[j]], steps):
                return True
    return False


def shared(written, read) -> bool:
    """Whether a view of `written` has a byte in common with another one or with one of `read`
    (or the search for it is too long to say that it has not)."""
    views = [(*v, True) for v in written] + [(*v, False) for v in read]
    spans = []
    for i, (at, levels, size, _) in enumerate(views):
        end = at + size
        for s, n in levels:
            end += s * n
        spans.append((at, end, i))
    steps = [_STEPS]
    try:
        return any(_share(views, g, None, steps) for g in _groups(spans))
    except _Undecided:
        return True
