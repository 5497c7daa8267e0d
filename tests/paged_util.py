"""Plain references of the paged cache's bookkeeping (whole numbers, one request at a time) and seeded states."""
import random


def free_pages(refs):
    return [p for p, n in enumerate(refs) if n == 0]


def plan(lens, new, table, refs, page, max_rows):
    """(lens, table, refs, cu_rows, slot_map, row_seq, row_pos, status) after mtp_page_plan."""
    slots, stride, free = len(lens), len(table[0]), free_pages(refs)
    none = (list(lens), [list(r) for r in table], list(refs), [0] * (slots + 1), [-1] * max_rows, [-1] * max_rows,
            [-1] * max_rows)
    if any(n < 0 or a < 0 or n + a > stride * page for n, a in zip(lens, new)) or sum(new) > max_rows:
        return (*none, [-1, 0, 0, len(free)])
    need = sum(-(-(n + a) // page) - -(-n // page) for n, a in zip(lens, new))
    if need > len(free):
        return (*none, [-2, 0, 0, len(free)])
    table, refs = [list(r) for r in table], list(refs)
    cu, places, seqs, poss, left = [0], [], [], [], iter(free)
    for s, (n, a) in enumerate(zip(lens, new)):
        for c in range(-(-n // page), -(-(n + a) // page)):
            table[s][c] = next(left)
            refs[table[s][c]] = 1
        for pos in range(n, n + a):
            held = table[s][pos // page]
            places.append(held * page + pos % page if 0 <= held < len(refs) else -1)
            seqs.append(s)
            poss.append(pos)
        cu.append(len(places))
    pad = [-1] * (max_rows - len(places))
    return ([n + a for n, a in zip(lens, new)], table, refs, cu, places + pad, seqs + pad, poss + pad,
            [0, len(seqs), need, len(free) - need])


def reorder(parent, table, lens, refs, page):
    """(table, lens, refs, copies [(from, to, rows)], status) after mtp_beam_reorder."""
    beams, stride, n_pages, free = len(parent[0]), len(table[0]), len(refs), free_pages(refs)
    bad = any(p >= beams for row in parent for p in row) or any(n < 0 or n > stride * page for n in lens)
    bad = bad or any(not 0 <= p < n_pages or refs[p] < 1 for r, n in zip(table, lens) for p in r[:-(-n // page)])
    if bad:
        return [list(r) for r in table], list(lens), list(refs), [], [-1, 0, len(free), 0]
    new_table, new_lens, copies = [], [], []
    for b, row in enumerate(parent):
        for j, p in enumerate(row):
            n = lens[b * beams + p] if p >= 0 else 0
            pages = list(table[b * beams + p][:-(-n // page)]) if p >= 0 else []
            if n % page and p in row[:j]:
                copies.append((pages[-1], len(copies), n % page))
                pages[-1] = ("fresh", len(copies) - 1)
            new_table.append(pages)
            new_lens.append(n)
    if len(copies) > len(free):
        return [list(r) for r in table], list(lens), list(refs), [], [-2, 0, len(free), 0]
    new_table = [[free[p[1]] if isinstance(p, tuple) else p for p in r] for r in new_table]
    copies = [(a, free[i], n) for a, i, n in copies]
    refs = list(refs)
    for r in new_table:
        for p in r:
            refs[p] += 1
    for r, n in zip(table, lens):
        for p in r[:-(-n // page)]:
            refs[p] -= 1
    return ([r + [-1] * (stride - len(r)) for r in new_table], new_lens, refs, copies,
            [0, len(copies), len(free_pages(refs)), 0])


def beams_state(seed, batch, beams, page, len_lo, len_hi, spare):
    """Tables, lengths and counts of `batch` items whose beams share a beginning of full pages."""
    rng = random.Random(seed)
    lens = [rng.randint(len_lo, len_hi) for _ in range(batch)]
    shared = [rng.randint(0, n // page) for n in lens]
    total = sum(beams * (-(-n // page) - s) + s for n, s in zip(lens, shared))
    n_pages = total + spare
    order = iter(rng.sample(range(n_pages), total))
    stride = -(-len_hi // page) + 2
    refs, table = [0] * n_pages, []
    for n, s in zip(lens, shared):
        common = [next(order) for _ in range(s)]
        for _ in range(beams):
            pages = common + [next(order) for _ in range(-(-n // page) - s)]
            for p in pages:
                refs[p] += 1
            table.append(pages + [rng.randint(-5, n_pages + 5) for _ in range(stride - len(pages))])  # unused: anything
    return table, [n for n in lens for _ in range(beams)], refs
