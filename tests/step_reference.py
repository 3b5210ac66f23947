"""Plain forms of a serving step in 64 bits on the CPU: page plan in integers, rotary positions, causal attention."""
import numpy as np
import torch

# half a unit in the last place, relative, of each storage type: 8, 11 and 24 significant bits
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def page_plan(kv, new, held, table, free, free_count, page_size, n_tokens):
    """Request after request, page after page.  Returns a dict of what ls_page_plan writes."""
    batch, width = table.shape
    table, free = table.copy(), free.copy()
    n_pages = len(free)
    cu = np.concatenate([[0], np.cumsum(np.maximum(new, 0).astype(np.int64))])
    err = np.zeros(batch, np.int32)
    for b in range(batch):
        want = -(-(int(kv[b]) + int(new[b])) // page_size)
        if kv[b] < 0 or new[b] < 0 or held[b] < 0 or held[b] > width or want > width or held[b] * page_size < kv[b] or \
                (n_tokens and cu[b + 1] > n_tokens):
            err[b] = 2
    stack = [int(p) for p in free[:free_count]]
    new_held = held.copy()
    for b in range(batch):
        want = -(-(int(kv[b]) + int(new[b])) // page_size)
        if not err[b] and want < held[b]:
            stack += [int(p) for p in table[b, want:held[b]]]
            new_held[b] = want
    free[free_count:len(stack)] = stack[free_count:]
    full = False
    for b in range(batch):
        want = -(-(int(kv[b]) + int(new[b])) // page_size)
        if err[b] or want <= held[b]:
            continue
        full = full or want - held[b] > len(stack)
        if full:
            err[b] = 1
            continue
        for i in range(held[b], want):
            table[b, i] = stack.pop()
        new_held[b] = want
    slots, positions = np.full(n_tokens, -1, np.int32), np.zeros(n_tokens, np.int32)
    for b in range(batch):
        for i in range(max(0, int(new[b]))):
            t = cu[b] + i
            if t >= n_tokens:
                break
            row = int(kv[b]) + i
            positions[t] = row
            if not err[b]:
                page = int(table[b, row // page_size])
                slots[t] = page * page_size + row % page_size if 0 <= page < n_pages else -1
    return {"table": table, "free": free, "new_held": new_held, "free_count": len(stack), "cu": cu.astype(np.int32),
            "total": np.where(err > 0, 0, kv + new).astype(np.int32), "slots": slots, "positions": positions, "err": err}


def rope(x, positions, cos_sin, sections, interleaved):
    """x [tokens, heads, head_dim] float64, positions [axes, tokens], cos_sin [rows, rotary_dim] -> (result, error scale of each
    element: the sum of the magnitudes of its two products)."""
    pairs = cos_sin.shape[1] // 2
    out, scale = x.copy(), np.zeros_like(x)
    pair = 0
    for axis, n in enumerate(sections):
        p = np.clip(positions[axis], 0, len(cos_sin) - 1)
        for i in range(pair, pair + n):
            c, s = cos_sin[p, i].astype(np.float64)[:, None], cos_sin[p, pairs + i].astype(np.float64)[:, None]
            e0, e1 = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
            a, b = x[:, :, e0], x[:, :, e1]
            out[:, :, e0], scale[:, :, e0] = a * c - b * s, np.abs(a * c) + np.abs(b * s)
            out[:, :, e1], scale[:, :, e1] = a * s + b * c, np.abs(a * s) + np.abs(b * c)
        pair += n
    return out, scale


def rope_bound(result, scale, dtype):
    """Two fp32 products and their sum: three roundings of at most 2^-24 of the magnitudes; then the storage type's."""
    return 3 * 2.0 ** -24 * scale + (HALF_ULP[dtype] if dtype != "f32" else 0.0) * np.abs(result) * 1.01 + 2.0 ** -40 + \
        (2.0 ** -25 if dtype == "f16" else 0.0)


def chunk_attention(q, k_rows, v_rows, news, lens, window, scale, dtype):
    """q [tokens, hq, d]; k_rows / v_rows: per request [hkv, rows, d]; all float64 (values exact in dtype).
    Returns out, lse and elementwise bounds of what the kernel's arithmetic may be off:
      scores      fp32 products and sums: (d + 8) 2^-24 of the sum of magnitudes (eps_s, largest over the row), and the
                  exponential, 4 * 2^-24 of the exponent in base 2 and 2^-22 of the value
      numerators  rounded to the storage type: half an ulp each; halves below 2^-14 of the largest: 2^-25 each
      the sum and the product: fp32, (rows + 64) 2^-24 at most, far less where tiles are added up
      the result rounded once more."""
    tokens, hq, d = q.shape
    out, lse = torch.zeros((tokens, hq, d), dtype=torch.float64), torch.full((tokens, hq), -torch.inf, dtype=torch.float64)
    out_bound, lse_bound = torch.zeros_like(out), torch.zeros_like(lse)
    at, half = 0, HALF_ULP[dtype]
    for n, kv, k, v in zip(news, lens, k_rows, v_rows):
        if n == 0:
            continue
        group = hq // k.shape[0]
        place = kv - n + torch.arange(n)[:, None]
        row = torch.arange(kv)[None]
        seen = (row <= place) & ((row > place - window) if window else torch.ones((1, 1), dtype=torch.bool))
        some = seen.any(1)
        for h in range(hq):
            if kv == 0 or not bool(some.any()):
                continue
            qh, kh, vh = q[at:at + n, h], k[h // group], v[h // group]
            s = torch.where(seen, qh @ kh.T * scale, -torch.inf)
            sizes = torch.where(seen, qh.abs() @ kh.abs().T * scale, 0.0)
            z = torch.logsumexp(s, 1, keepdim=True)
            w = torch.where(some[:, None], torch.exp(s - z), 0.0)
            eps = ((d + 8) * 2.0 ** -24 * sizes.amax(1) + 8 * 2.0 ** -24 * torch.where(seen, s, 0.0).abs().amax(1) + 2.0 ** -22)[:, None]
            magnitude = w @ vh.abs()
            summed = (kv + 64) * 2.0 ** -24
            small = 2.0 ** -25 * seen.double() @ vh.abs() / torch.exp(z - s.amax(1, keepdim=True)).clamp(min=1) if dtype == "f16" else 0.0
            o = w @ vh
            ok = slice(at, at + n)
            out[ok, h] = torch.where(some[:, None], o, 0.0)
            lse[ok, h] = torch.where(some, z[:, 0], -torch.inf)
            bound = 1.02 * ((half + 2 * eps + 2 * summed) * magnitude + small + half * o.abs()) + (2.0 ** -25 if dtype == "f16" else 2.0 ** -130)
            out_bound[ok, h] = torch.where(some[:, None], torch.nan_to_num(bound, nan=0.0), 0.0)
            lse_bound[ok, h] = torch.where(some, eps[:, 0] + summed + 4 * 2.0 ** -24 * z[:, 0].abs(), 0.0)
        at += n
    return out, lse, out_bound, lse_bound
