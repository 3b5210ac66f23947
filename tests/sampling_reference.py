"""Plain implementations of the operators of sampled decoding, on the CPU: the verification by its definition, distribution by
distribution in more than 64 bits, and the tables' operators request by request on lists."""
import numpy as np

FLT_MAX = float(np.finfo(np.float32).max)


def softmax(row, temperature, largest=FLT_MAX):
    """Weights and their sum to 1 (or all 0), and the log probabilities; -inf and NaN have none, +inf is the largest finite number."""
    x = np.asarray(row, dtype=np.longdouble).copy()
    x[np.isnan(x)] = -np.inf
    x[x == np.inf] = largest
    top = x.max()
    if top == -np.inf:
        return np.zeros_like(x), np.full_like(x, -np.inf)
    with np.errstate(under="ignore", invalid="ignore", divide="ignore"):
        y = np.where(x == -np.inf, -np.inf, (x - top) / np.longdouble(temperature))
        w = np.exp(y)
        return w / w.sum(), y - np.log(w.sum())


def accept_sampled(parents, tokens, target, draft, temperature, draft_temperature, accept_u, sample_u, with_replacement,
                   largest=(FLT_MAX, FLT_MAX)):
    """One sequence.  target, draft: arrays [n_tree, vocab] (draft None: chosen); largest: finite number of their types.  Returns path, next token, log probabilities, error."""
    n, vocab = target.shape
    err, above = 0, list(parents)
    for i, p in enumerate(above):
        if p < -1 or p >= i:
            above[i], err = -1, 1
    heats = []
    for t in (temperature, temperature if draft_temperature is None else draft_temperature):
        t = float(t)
        if not 0 <= t <= FLT_MAX:
            err |= 2
            t = 0.0
        heats.append(t)
    path, logs = [0], []
    while True:
        cur = path[-1]
        p, log_p = softmax(target[cur], heats[0] or 1.0, largest[0])
        if heats[0] == 0:
            best = int(np.argmax(p)) if p.any() else -1
            p = np.zeros_like(p)
            if best >= 0:
                p[best] = 1
        kids = [i for i in range(n) if above[i] == cur and i > cur and 0 <= tokens[i] < vocab]
        drawn = draft is not None and heats[0] > 0 and heats[1] > 0
        q = softmax(draft[cur], heats[1], largest[1])[0] if drawn and kids else None
        found = None
        for k in kids:
            x = tokens[k]
            # u < p / q, also where q is 0
            if (p[x] > np.longdouble(accept_u[k]) * q[x]) if drawn else p[x] > accept_u[k]:
                found = k
                break
            if drawn:
                p = np.maximum(p - q, 0)
                p[x] = 0
                if not with_replacement:
                    q[x] = 0
                    if q.sum() > 0:
                        q = q / q.sum()
            else:
                p[x] = 0
            if p.sum() > 0:
                p = p / p.sum()
        if found is not None:
            path.append(found)
            logs.append(log_p[tokens[found]])
            continue
        if not p.sum() > 0:
            return path, -1, logs + [-np.inf], err | 4
        upto = np.cumsum(p)
        passed = np.flatnonzero(upto > np.longdouble(sample_u) * upto[-1])
        token = int(passed[0]) if len(passed) else int(np.flatnonzero(p)[-1])
        return path, token, logs + [log_p[token]], err


def fork(sources, keep_lens, kv_lens, held, table, free, count, page_size, n_pages):
    """Lists; table: a list of rows.  Returns the new rows (entries held), kv_lens, held, free (a copy), count, copies, err."""
    batch, stride = len(sources), len(table[0])
    clamp = lambda v, lo, hi: max(lo, min(hi, v))  # noqa: E731
    goes = []
    for b, s in enumerate(sources):
        if s == -1:
            goes.append((b, 0, 0, 0, 0))
            continue
        if 0 <= s < batch:
            c, h = kv_lens[s], held[s]
            keep = c if keep_lens is None else keep_lens[b]
            if c >= 0 and 0 <= h <= stride and h * page_size >= c and 0 <= keep <= c:
                goes.append((s, keep, keep // page_size, keep % page_size, 0))
                continue
        h = clamp(held[b], 0, stride)
        goes.append((b, clamp(kv_lens[b], 0, h * page_size), h, 0, 2))
    inside = lambda p: 0 <= p < n_pages  # noqa: E731
    as_full = {p for s, _, full, _, _ in goes for p in table[s][:full] if inside(p)}
    heir = {}
    for b, (s, _, full, part, _) in enumerate(goes):
        if part:
            heir.setdefault(table[s][full], b)
    kept = set(as_full) | {p for p in heir if inside(p)}
    free, stack, seen = list(free), list(free[:clamp(count, 0, n_pages)]), set()
    for b in range(batch):
        for p in table[b][:clamp(held[b], 0, stride)]:
            if inside(p) and p not in kept and p not in seen:
                seen.add(p)
                stack.append(p)
    for i in range(clamp(count, 0, n_pages), min(len(stack), n_pages)):
        free[i] = stack[i]
    rows, lens, new_held, copies, errs = [], [], [], [], []
    for b, (s, keep, full, part, err) in enumerate(goes):
        row = list(table[s][:full])
        if part:
            page = table[s][full]
            if not inside(page) or (page not in as_full and heir[page] == b):
                row.append(page)
            elif stack:
                fresh = stack.pop()
                copies.append((page, fresh, part, b))
                row.append(fresh)
            else:
                keep, err = full * page_size, 1
        rows.append(row)
        lens.append(keep)
        new_held.append(len(row))
        errs.append(err)
    return rows, lens, new_held, free, min(len(stack), n_pages), copies, errs


def compact(held, table, page_size, n_pages):
    """Returns the new rows, the stack of free pages, copies."""
    rows = [row[:max(0, min(len(row), h))] for row, h in zip(table, held)]
    used = sorted({p for row in rows for p in row if 0 <= p < n_pages})
    n = len(used)
    holes = iter(sorted(set(range(n)) - set(used)))
    moved = {p: next(holes) for p in used if p >= n}
    return [[moved.get(p, p) for p in row] for row in rows], list(range(n_pages - 1, n - 1, -1)), [(p, q, page_size, -1) for p, q in moved.items()]
