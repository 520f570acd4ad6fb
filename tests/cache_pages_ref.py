"""Fork, trim and compact of the paged KV cache in plain Python, one page after the other, written from the definitions
in include/rotate_attn.h.  A state is a dict of seq, table (lists of lists), refs, free (a list of num_pages), count and
cache (a list of page contents)."""
import copy


def up(n, page):
    return -(-n // page)


def valid(state, page):
    """What holds between the tables of a sound state: holders, stack and tables agree."""
    pages = len(state["refs"])
    held = [0] * pages
    for n, row in zip(state["seq"], state["table"]):
        for id in row[:up(n, page)]:
            if id >= 0:
                held[id] += 1
    stack = state["free"][:state["count"]]
    assert len(set(stack)) == len(stack) and all(0 <= x < pages for x in stack)
    for id in range(pages):
        assert (held[id] == 0) == (id in stack), id
        assert state["refs"][id] == max(0, held[id] - 1), id


def _is(id, pages):
    return 0 <= id < pages


def fork(state, page, max_blocks, parents, children, lens=None):
    """(state afterwards, status)."""
    s, R, pages = copy.deepcopy(state), len(state["seq"]), len(state["refs"])
    flags, taken = 0, 0
    for i, (a, c) in enumerate(zip(parents, children)):
        if not (0 <= a < R and 0 <= c < R):
            flags |= 1
            continue
        n = state["seq"][a]
        L = n if lens is None else lens[i]
        if c in children[:i] or state["seq"][c] != 0 or not 0 <= n <= max_blocks * page or not 0 <= L <= n:
            flags |= 1
        taken += L % page > 0
    if not 0 <= state["count"] <= pages:
        flags |= 8
    elif taken > state["count"]:
        flags |= 4
    if flags:
        return s, flags
    shared = 0
    for i, (a, c) in enumerate(zip(parents, children)):
        L = state["seq"][a] if lens is None else lens[i]
        for j in range(L // page):
            id = state["table"][a][j]
            s["table"][c][j] = id
            if _is(id, pages):
                s["refs"][id] += 1
                shared += 1
        if L % page:
            s["count"] -= 1
            new, old = s["free"][s["count"]], state["table"][a][L // page]
            s["table"][c][L // page] = new
            if _is(old, pages):
                s["cache"][new] = state["cache"][old]
        s["seq"][c] = L
    return s, [0, taken, shared, max([0] + s["seq"])]


def trim(state, page, max_blocks, window, keep=None, sinks=-1):
    s, R, pages = copy.deepcopy(state), len(state["seq"]), len(state["refs"])
    flags, need, kept = 0, 0, []
    for r in range(R):
        n = state["seq"][r]
        k = n if keep is None or keep[r] < 0 else keep[r]
        kept.append(k)
        if not 0 <= n <= max_blocks * page or k > n:
            flags |= 1
        elif k % page:
            id = state["table"][r][k // page]
            need += _is(id, pages) and state["refs"][id] > 0
    if not 0 <= state["count"] <= pages:
        flags |= 8
    elif need > state["count"]:
        flags |= 4
    if flags:
        return s, flags
    lost = [0] * pages

    def go(r, j):
        id = state["table"][r][j]
        if _is(id, pages):
            lost[id] += 1
        s["table"][r][j] = -1

    for r in range(R):
        n, k = state["seq"][r], kept[r]
        if k % page:
            id = state["table"][r][k // page]
            if _is(id, pages) and state["refs"][id] > 0:
                s["count"] -= 1
                new = s["free"][s["count"]]
                s["table"][r][k // page] = new
                s["cache"][new] = state["cache"][id]
                lost[id] += 1
        for j in range(up(k, page), up(n, page)):
            go(r, j)
        if sinks >= 0:
            for j in range(up(k, page)):
                if j * page >= sinks and (j + 1) * page <= k - window + 1:
                    go(r, j)
        s["seq"][r] = k
    back = 0
    for id in range(pages):
        if lost[id] > s["refs"][id]:
            s["free"][s["count"]] = id
            s["count"] += 1
            s["refs"][id] = 0
            back += 1
        else:
            s["refs"][id] -= lost[id]
    return s, [0, need, back, max([0] + kept)]


def compact(state, page, max_blocks):
    s, pages = copy.deepcopy(state), len(state["refs"])
    flags = 0
    if any(not 0 <= n <= max_blocks * page for n in state["seq"]):
        flags |= 1
    if not 0 <= state["count"] <= pages:
        return s, flags | 8
    stack = state["free"][:state["count"]]
    if len(set(stack)) < len(stack) or not all(_is(x, pages) for x in stack):
        flags |= 16
    if flags:
        return s, flags
    k = pages - state["count"]
    src = [i for i in range(k, pages) if i not in set(stack)]
    dst = sorted(i for i in stack if i < k)
    to = dict(zip(src, dst))
    for a, b in to.items():
        s["cache"][b] = state["cache"][a]
        s["refs"][b] = state["refs"][a]
        s["refs"][a] = 0
    for r, n in enumerate(state["seq"]):
        for j in range(up(n, page)):
            s["table"][r][j] = to.get(s["table"][r][j], s["table"][r][j])
    for i in range(state["count"]):
        s["free"][i] = pages - 1 - i
    return s, [0, len(to), k, 0]
