"""Operators around the pruned cache, as cases that can be timed and compared: in plain torch, or by the framework's calls.

Four kinds of pass:

  rotary  queries and keys get their rotary positions as the projection leaves them; the keys (and values) go to the layout
          that the pruning and caching calls take, as bf16 or as 8-bit rows
  fork    sequences of the cache become copies of others (beams, best of n), and their lists are handed over as packed rows
  move    sequences come in as packed rows, go into the cache's pages and windows, and are packed again
  attend  the new token's attention for groups of sequences that share a long prefix: forked, then decoded for some steps

Sizes: 8 KV heads of 128, 32 query heads, pages of 16 rows, window 128 and about a quarter of a context kept, as the models of
the benchmark have them, and odd ones beside them.
"""
import math
import random

import torch

own = False

H = 8                      # KV heads
MINUS_INF = float("-inf")


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # One new token for each of 8 sequences: latency.
        _rotary("rotary_decode_b8", tokens=8, top=32768),
        # A 32k prompt, frequencies scaled for a longer context, keys to the head-major layout of the pruning calls.
        _rotary("rotary_prompt_32k", tokens=32768, top=32768, factor=8.0, head_major=True),
        # Chunks of several prompts, half of each head rotated, neighbouring pairs, positions past 2^20.
        _rotary("rotary_half_head_7777", tokens=7777, rotary=64, interleaved=True, top=4000000, factor=32.0),
        # A prompt for an 8-bit cache: keys and values become rows of codes with a scale.
        _rotary("rotary_rows8_16411", tokens=16411, top=131072, head_major=True, rows8=True),
        # Three beams from one short sequence, two layers: latency.
        _fork("fork_3_short", layers=2, sources=1, children=3, rows=200, steps=20),
        # Two prompts of 8k tokens, seven samples of each, a block of layers.
        _fork("fork_2x7", layers=12, sources=2, children=7, rows=2000, steps=128),
        # One short sequence of a few layers swapped in and out.
        _move("move_1_short", layers=4, seqs=1, rows=300, tokens=61),
        # Two preempted sequences of a whole model.
        _move("move_2_36l", layers=36, seqs=2, rows=2000, tokens=500),
        # Four samples of a short prompt, one layer: latency.
        _attend("attend_4x1k", layers=1, groups=1, members=4, rows=1000, steps=20),
        # A system prompt of 32k tokens under 32 conversations, a block of layers.
        _attend("attend_32x8k_4l", layers=4, groups=1, members=32, rows=8000, steps=150),
        # Two documents of 128k tokens, 64 questions about each.
        _attend("attend_2x64x32k", layers=2, groups=2, members=64, rows=32768, steps=300),
        # Odd sizes: 64 elements a head, 7 query heads for each KV head, pages of 48 rows, three groups of 5.
        _attend("attend_3x5_odd", layers=12, groups=3, members=5, rows=2345, steps=77, dim=64, per_kv=7, page=48, window=48),
    ]


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "fork", "move", "attend", "attend", "attend"])
    if kind == "rotary":
        dim = rng.choice([64, 128, 128])
        return _rotary(None, tokens=_log(rng, 1, 32768), dim=dim, per_kv=rng.choice([1, 2, 4, 5, 8]),
                       rotary=rng.choice([dim, dim, dim // 2, dim // 4]), interleaved=rng.random() < 0.4,
                       top=_log(rng, 100, 8000000), factor=rng.choice([1.0, 1.0, 4.0, 32.0]), head_major=rng.random() < 0.5,
                       rows8=rng.random() < 0.3, inverse=rng.random() < 0.2)
    layers = rng.choice([1, 2, 4, 12])
    if kind == "fork":
        sources = rng.choice([1, 1, 2, 3])
        children = _log(rng, 1, 16 // sources)
        return _fork(None, layers=layers, sources=sources, children=children, rows=_log(rng, 20, 4000 // sources),
                     steps=rng.randint(1, 128), page=rng.choice([16, 16, 32, 128]))
    if kind == "move":
        seqs = _log(rng, 1, 8)
        return _move(None, layers=layers, seqs=seqs, rows=_log(rng, 20, 12000 // seqs), tokens=rng.randint(1, 1000),
                     page=rng.choice([16, 16, 32, 128]))
    groups = rng.choice([1, 1, 2, 3])
    members = _log(rng, 2, 64 // groups)
    return _attend(None, layers=rng.choice([1, 1, 2, 4]), groups=groups, members=members,
                   rows=_log(rng, 100, 32768 // groups), steps=rng.randint(1, 300), dim=rng.choice([64, 128, 128]),
                   per_kv=rng.choice([1, 2, 4, 4, 5, 8]), page=rng.choice([16, 16, 32, 48, 128]),
                   window=rng.choice([32, 128, 128, 256]))


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def _named(name, case):
    return dict(case, name=name) if name else case


def _rotary(name, tokens, top, dim=128, per_kv=4, rotary=None, interleaved=False, factor=1.0, head_major=False, rows8=False,
            inverse=False):
    return _named(name, {"kind": "rotary", "tokens": tokens, "top": top, "dim": dim, "per_kv": per_kv,
                         "rotary": rotary or dim, "interleaved": interleaved, "factor": factor, "head_major": head_major,
                         "rows8": rows8, "inverse": inverse})


def _fork(name, layers, sources, children, rows, steps, page=16, dim=128, window=128):
    return _named(name, {"kind": "fork", "layers": layers, "sources": sources, "children": children, "rows": rows,
                         "steps": steps, "page": page, "dim": dim, "window": window})


def _move(name, layers, seqs, rows, tokens, page=16, dim=128, window=128):
    return _named(name, {"kind": "move", "layers": layers, "seqs": seqs, "rows": rows, "tokens": tokens, "page": page,
                         "dim": dim, "window": window})


def _attend(name, layers, groups, members, rows, steps, dim=128, per_kv=4, page=16, window=128):
    return _named(name, {"kind": "attend", "layers": layers, "groups": groups, "members": members, "rows": rows,
                         "steps": steps, "dim": dim, "per_kv": per_kv, "page": page, "window": window})


# --------------------------------------------------------------------------------------------------------------- inputs

def _gen(seed, *at):
    for a in at:
        seed = (seed * 1000003 + 7919 * (a + 1)) % (1 << 48)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(gen, *shape):
    return torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _lengths(case, n_lists):
    """Rows of each pruned list: about case["rows"], spread over 1 : 5 by head, never empty."""
    rng = random.Random("lengths %d %d" % (case["rows"], n_lists))
    return [max(1, int(case["rows"] * rng.uniform(0.35, 1.65))) for _ in range(n_lists)]


def _int(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _tables(counts, page, width, gen):
    """Page numbers of lists of so many rows, handed out in a random order from page 0 on: (table, pages handed out)."""
    need = [-(-n // page) for n in counts]
    order = torch.randperm(sum(need), generator=gen, device="cuda").to(torch.int32)
    n = _int(need, torch.int64)
    at = torch.cumsum(n, 0) - n
    col = torch.arange(width, device="cuda")
    index = (at[:, None] + col).clamp(max=sum(need) - 1)
    return torch.where(col < n[:, None], order[index], torch.zeros((), dtype=torch.int32, device="cuda")), sum(need)


class _Session:
    """A program's context and cache; freed with the object, the cache first."""

    def __init__(self, layers, dim, max_tokens, rows8=False):
        from paper_2601_07891_b200 import binding
        self.cache = None
        self.ctx = binding.Kvzap(64, 0, H, (dim + 16) // 2 if rows8 else dim, layers, max_tokens=max_tokens)

    def open_cache(self, n_seqs, case, K_pool, V_pool, width):
        self.cache = self.ctx.create_cache(n_seqs, case["window"], case["page"], K_pool, V_pool, width)

    def __del__(self):
        try:
            if self.cache is not None:
                self.cache.close()
            self.ctx.close()
        except Exception:                           # the interpreter is going down
            pass


def prepare(case, seed):
    s = {"rotary": _prepare_rotary, "fork": _prepare_fork, "move": _prepare_move, "attend": _prepare_attend}[case["kind"]](case, seed)
    s["case"] = case
    return s


def run(s):
    return {"rotary": _run_rotary, "fork": _run_fork, "move": _run_move, "attend": _run_attend}[s["case"]["kind"]](s)


def work(case):
    return {"rotary": _work_rotary, "fork": _work_fork, "move": _work_move, "attend": _work_attend}[case["kind"]](case)


def exact(case, seed):
    return {"rotary": _exact_rotary, "fork": _exact_fork, "move": _exact_move, "attend": _exact_attend}[case["kind"]](case, seed)


# --------------------------------------------------------------------------------------------------------------- rotary

ROTARY_BASE = 500000.0
CONTEXT = 8192                                      # scaled frequencies: the context that the model was trained with
LOW, HIGH = 1.0, 4.0                                # ... turns in it below / above which a pair is scaled / left alone


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["interleaved"] else 1.0


def _rotary_inputs(case, seed):
    """A fused projection's rows (queries, keys, values of a token side by side) and the tokens' positions."""
    T, D = case["tokens"], case["dim"]
    n_q = H * case["per_kv"]
    qkv = _normal(_gen(seed, 0), T, n_q + 2 * H, D)
    positions = torch.randint(0, case["top"], (T,), generator=_gen(seed, 1), device="cuda", dtype=torch.int32)
    return qkv[:, :n_q], qkv[:, n_q:n_q + H], qkv[:, n_q + H:], positions


def _prepare_rotary(case, seed):
    Q, K, V, positions = _rotary_inputs(case, seed)
    T, D = case["tokens"], case["dim"]
    s = {"Q": Q, "K": K, "V": V, "positions": positions}
    if own:
        s["session"] = _Session(1, D, 64, case["rows8"])
        s["session"].ctx.set_rotary(rotary_dim=case["rotary"], head_dim=D, base=ROTARY_BASE, interleaved=case["interleaved"],
                                    factor=case["factor"], original_context=CONTEXT, low=LOW, high=HIGH,
                                    magnitude=_magnitude(case))
        shape = (H, T) if case["head_major"] else (T, H)

        def rows():
            r = torch.empty(*shape, D + 16, dtype=torch.uint8, device="cuda") if case["rows8"] else \
                torch.empty(*shape, D, dtype=torch.bfloat16, device="cuda")
            return r.transpose(0, 1) if case["head_major"] else r

        s["Q_out"] = torch.empty(T, H * case["per_kv"], D, dtype=torch.bfloat16, device="cuda")
        s["K_out"] = rows()
        s["V_out"] = rows() if case["rows8"] else None
    return s


def _frequencies(case):
    R = case["rotary"]
    f = ROTARY_BASE ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R)
    turns = CONTEXT * f / (2 * math.pi)
    keep = ((turns - LOW) / (HIGH - LOW)).clamp(0, 1)
    return (1 - keep) * f / case["factor"] + keep * f


def _codes(x):
    """8-bit rows of fp32 rows: E4M3 codes whose largest stands for 448 scales, and the scales."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.where(top > 0, top / 448.0, torch.ones_like(top))
    return (x / scale).to(torch.float8_e4m3fn), scale


def _run_rotary(s):
    case = s["case"]
    R, D = case["rotary"], case["dim"]
    if own:
        s["session"].ctx.rotary(s["positions"], s["Q"], s["K"], s["V"] if case["rows8"] else None, Q_out=s["Q_out"],
                                K_out=s["K_out"], V_out=s["V_out"], inverse=case["inverse"])
        out = [s["Q_out"]]
        for t in (s["K_out"], s["V_out"]) if case["rows8"] else (s["K_out"],):
            t = t.transpose(0, 1) if case["head_major"] else t
            out += [t[..., :D].view(torch.float8_e4m3fn), t[..., D:D + 4].view(torch.float32)] if case["rows8"] else [t]
        return out
    angle = s["positions"].double()[:, None] * _frequencies(case)
    sign = -1.0 if case["inverse"] else 1.0
    cos = (angle.cos() * _magnitude(case)).float()[:, None]
    sin = (angle.sin() * (sign * _magnitude(case))).float()[:, None]

    def rotated(x):
        x = x.float()
        y = x.clone()
        a, b = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y

    out = [rotated(s["Q"]).bfloat16()]
    for t in (rotated(s["K"]), s["V"].float()) if case["rows8"] else (rotated(s["K"]),):
        t = t.transpose(0, 1).contiguous() if case["head_major"] else t
        out += list(_codes(t)) if case["rows8"] else [t.bfloat16()]
    return out


def _exact_rotary(case, seed):
    Q, K, V, positions = _rotary_inputs(case, seed)
    R = case["rotary"]
    inv = [ROTARY_BASE ** (-2.0 * i / R) for i in range(R // 2)]
    for i, f in enumerate(inv):
        wavelength = 2 * math.pi / f
        part = min(1.0, max(0.0, (CONTEXT / wavelength - LOW) / (HIGH - LOW)))
        inv[i] = f * (part + (1.0 - part) / case["factor"])
    angle = torch.outer(positions.double(), _int(inv, torch.float64))
    turn = torch.polar(torch.full_like(angle, _magnitude(case)), -angle if case["inverse"] else angle)[:, None]
    out = []
    for x, turns in ((Q, True), (K, True), (V, False)):
        x = x.double()
        if turns:
            z = x[..., :R]
            z = z.unflatten(-1, (R // 2, 2)) if case["interleaved"] else z.unflatten(-1, (2, R // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            z = z if case["interleaved"] else z.transpose(-1, -2)
            x = torch.cat([z.flatten(-2), x[..., R:]], -1)
        out.append(x)
    rows = [t.transpose(0, 1) if case["head_major"] else t for t in out[1:]]
    if not case["rows8"]:
        return [out[0], rows[0]]
    full = [out[0]]
    for t in rows:
        scale = t.abs().amax(-1, keepdim=True) / 448.0
        full += [(t / scale).float().to(torch.float8_e4m3fn).double(), scale]
    return full


def _work_rotary(case):
    T, D, n_q = case["tokens"], case["dim"], H * case["per_kv"]
    read = T * (n_q + H * (2 if case["rows8"] else 1)) * D * 2 + 4 * T
    write = T * n_q * D * 2 + (T * 2 * H * (D + 16) if case["rows8"] else T * H * D * 2)
    return {"bytes": read + write, "flops": 3 * T * (n_q + H) * case["rotary"]}


# ----------------------------------------------------------------------------------------------------- lists of the cache

def _pack_plain(K_pool, V_pool, table, prefix, K_ring, V_ring, scores, tokens, page):
    """The rows of lists (pages first, then the window, oldest first), one list after the other; [n] lists."""
    w, D = K_ring.shape[1:]
    prefix, tokens = prefix.long(), tokens.long()
    count = prefix + tokens.clamp(max=w)
    ends = torch.cumsum(count, 0)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), ends])
    which = torch.repeat_interleave(torch.arange(count.numel(), device="cuda"), count)
    r = torch.arange(which.numel(), device="cuda") - start[which]
    paged = r < prefix[which]
    at_page = table[which, (r // page).clamp(max=table.shape[1] - 1)].long() * page + r % page
    position = (tokens - tokens.clamp(max=w))[which] + r - prefix[which]
    at_ring = which * w + position % w
    rows = []
    for pool, ring in ((K_pool, K_ring), (V_pool, V_ring)):
        rows.append(torch.where(paged[:, None], pool.view(-1, D)[torch.where(paged, at_page, 0)],
                                ring.reshape(-1, D)[torch.where(paged, 0, at_ring)]))
    slot = torch.arange(w, device="cuda")
    first = (tokens - tokens.clamp(max=w))[:, None]
    kept = torch.where(slot < tokens.clamp(max=w)[:, None], torch.gather(scores, 1, (first + slot) % w), 0.0)
    return rows[0], rows[1], start, tokens.int(), kept


# ----------------------------------------------------------------------------------------------------------------- fork

def _fork_inputs(case, seed):
    """Sources in slots 0 .. n-1: paged prefixes, and a window of steps tokens; pools with room for what is forked."""
    S, L, D, steps = case["sources"], case["layers"], case["dim"], case["steps"]
    slots = S * (1 + case["children"])
    counts = _lengths(case, S * L * H)
    page = case["page"]
    width = -(-max(counts) // page) + 1
    table, used = _tables(counts, page, width, _gen(seed, 0))
    n_pages = used + slots * L * H
    K_pool, V_pool = (_normal(_gen(seed, 1 + i), n_pages, page, D) for i in range(2))
    K_new, V_new = (_normal(_gen(seed, 3 + i), steps, L, slots, H, D) for i in range(2))
    hidden = _normal(_gen(seed, 5), steps, L, slots, 64)
    W = _normal(_gen(seed, 6), L, H, 64) * 0.125
    return slots, counts, width, table, used, K_pool, V_pool, K_new, V_new, hidden, W


def _fork_pairs(case):
    S, n = case["sources"], case["children"]
    return [i // n for i in range(S * n)], list(range(S, S * (n + 1)))


def _prepare_fork(case, seed):
    slots, counts, width, table, used, K_pool, V_pool, K_new, V_new, hidden, W = _fork_inputs(case, seed)
    S, L, D, w, steps = case["sources"], case["layers"], case["dim"], case["window"], case["steps"]
    n_src, n_all = S * L * H, slots * L * H
    src, dst = _fork_pairs(case)
    total = sum((counts[s * L * H + i] + min(steps, w)) for s in src for i in range(L * H))
    full_table = torch.zeros(n_all, width, dtype=torch.int32, device="cuda")
    full_table[:n_src] = table
    prefix = torch.zeros(n_all, dtype=torch.int32, device="cuda")
    prefix[:n_src] = _int(counts)
    s = {"src": src, "dst": dst, "K_pool": K_pool, "V_pool": V_pool}
    if own:
        s["session"] = session = _Session(L, D, max(64, slots))
        for l in range(L):
            session.ctx.set_weights(l, W[l].contiguous(), None)
        session.open_cache(slots, case, K_pool, V_pool, width)
        session.cache.import_prefix(prefix, full_table, used)
        for t in range(steps):
            session.cache.decode_step(0, L, hidden[t], K_new[t], V_new[t], MINUS_INF)
        s["K_out"], s["V_out"] = (torch.empty(total, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return s
    s["table"], s["prefix"], s["spare"] = full_table, prefix, _int(range(used, used + n_all))
    for key, new in (("K_ring", K_new), ("V_ring", V_new)):
        ring = torch.zeros(n_all, w, D, dtype=torch.bfloat16, device="cuda")
        ring[:, :steps] = new.permute(2, 1, 3, 0, 4).reshape(n_all, steps, D)
        s[key] = ring
    s["scores"] = torch.zeros(n_all, w, device="cuda")
    scored = torch.einsum("tlbd,lhd->blht", hidden.float(), W.float())
    s["scores"][:, :steps] = scored.reshape(n_all, steps)
    s["tokens"] = torch.full((n_all,), steps, dtype=torch.int32, device="cuda")
    return s


def _run_fork(s):
    if own:
        cache = s["session"].cache
        cache.fork(s["src"], s["dst"])
        return cache.pack(s["dst"], K_out=s["K_out"], V_out=s["V_out"])
    case = s["case"]
    each, page = case["layers"] * H, case["page"]
    lists = torch.arange(each, device="cuda")
    src = (_int(s["src"], torch.int64)[:, None] * each + lists).flatten()
    dst = (_int(s["dst"], torch.int64)[:, None] * each + lists).flatten()
    whole = (s["prefix"][src] // page).long()
    s["table"][dst] = s["table"][src]
    last = s["table"][src, whole.clamp(max=s["table"].shape[1] - 1)].long()
    for pool in (s["K_pool"], s["V_pool"]):
        pool[s["spare"][dst].long()] = pool[last]
    s["table"][dst, whole] = s["spare"][dst]
    for key in ("prefix", "tokens", "K_ring", "V_ring", "scores"):
        s[key][dst] = s[key][src]
    return _pack_plain(s["K_pool"], s["V_pool"], s["table"][dst], s["prefix"][dst], s["K_ring"][dst], s["V_ring"][dst],
                       s["scores"][dst], s["tokens"][dst], page)


def _exact_fork(case, seed):
    slots, counts, width, table, used, K_pool, V_pool, K_new, V_new, hidden, W = _fork_inputs(case, seed)
    L, D, w, steps = case["layers"], case["dim"], case["window"], case["steps"]
    src, _ = _fork_pairs(case)
    K, V, kept, ends = [], [], [], [0]
    for b in src:
        for l in range(L):
            for h in range(H):
                i = (b * L + l) * H + h
                pages = table[i, :-(-counts[i] // case["page"])].long()
                for out, pool, new in ((K, K_pool, K_new), (V, V_pool, V_new)):
                    out.append(torch.cat([pool[pages].reshape(-1, D)[:counts[i]], new[:, l, b, h]]))
                score = torch.zeros(w, dtype=torch.float64, device="cuda")
                score[:steps] = hidden[:, l, b].double() @ W[l, h].double()
                kept.append(score)
                ends.append(ends[-1] + counts[i] + steps)
    return [torch.cat(K).double(), torch.cat(V).double(), _int(ends, torch.int64), _int([steps] * (len(ends) - 1)), torch.stack(kept)]


def _work_fork(case):
    S, n, L, D, w = case["sources"], case["children"], case["layers"], case["dim"], case["window"]
    rows = sum(_lengths(case, S * L * H)) * n
    window = S * n * L * H * min(case["steps"], w)
    # the window, half a page and the page table of each child are read and written, then all of its rows
    copied = S * n * L * H * (case["page"] // 2 + min(case["steps"], w)) * D * 4
    return {"bytes": 2 * copied + 2 * (rows + window) * D * 4, "flops": 0}


# ----------------------------------------------------------------------------------------------------------------- move

def _move_inputs(case, seed):
    """Packed lists: rows[i] rows of pages and the last min(tokens, window) of a sequence's tokens."""
    B, L, D, w = case["seqs"], case["layers"], case["dim"], case["window"]
    counts = _lengths(case, B * L * H)
    n_win = min(case["tokens"], w)
    ends = [0]
    for c in counts:
        ends.append(ends[-1] + c + n_win)
    K, V = (_normal(_gen(seed, 1 + i), ends[-1], D) for i in range(2))
    scores = torch.zeros(B * L * H, w, device="cuda")
    scores[:, :n_win] = torch.randn(B * L * H, n_win, generator=_gen(seed, 3), device="cuda")
    return counts, _int(ends, torch.int64), K, V, _int([case["tokens"]] * (B * L * H)), scores


def _prepare_move(case, seed):
    counts, start, K, V, tokens, scores = _move_inputs(case, seed)
    B, L, D, w, page = case["seqs"], case["layers"], case["dim"], case["window"], case["page"]
    n = B * L * H
    width = -(-max(counts) // page) + 1
    table, used = _tables(counts, page, width, _gen(seed, 0))
    K_pool, V_pool = (torch.zeros(used + 1, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s = {"K": K, "V": V, "start": start, "tokens": tokens, "scores": scores, "slots": list(range(B)), "K_pool": K_pool,
         "V_pool": V_pool}
    if own:
        s["session"] = _Session(L, D, max(64, B))
        s["session"].open_cache(B, case, K_pool, V_pool, width)
        s["K_out"], s["V_out"] = torch.empty_like(K), torch.empty_like(V)
        return s
    s["table"], s["prefix"] = table, torch.zeros(n, dtype=torch.int32, device="cuda")
    s["K_ring"], s["V_ring"] = (torch.zeros(n, w, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s["score_ring"] = torch.zeros(n, w, device="cuda")
    return s


def _run_move(s):
    if own:
        cache = s["session"].cache
        cache.unpack(s["slots"], s["K"], s["V"], s["start"], s["tokens"], s["scores"])
        return cache.pack(s["slots"], K_out=s["K_out"], V_out=s["V_out"])
    page, w, D = s["case"]["page"], s["case"]["window"], s["case"]["dim"]
    start, tokens = s["start"], s["tokens"].long()
    count = start[1:] - start[:-1]
    n_win = tokens.clamp(max=w)
    s["prefix"].copy_(count - n_win)
    which = torch.repeat_interleave(torch.arange(count.numel(), device="cuda"), count)
    r = torch.arange(which.numel(), device="cuda") - start[which]
    paged = r < s["prefix"][which]
    wl, rl = which[paged], r[paged]
    at_page = s["table"][wl, rl // page].long() * page + rl % page
    wr, rr = which[~paged], r[~paged]
    at_ring = wr * w + (tokens[wr] - n_win[wr] + rr - s["prefix"][wr]) % w
    for rows, pool, ring in ((s["K"], s["K_pool"], s["K_ring"]), (s["V"], s["V_pool"], s["V_ring"])):
        pool.view(-1, D)[at_page] = rows[paged]
        ring.view(-1, D)[at_ring] = rows[~paged]
    s["score_ring"].view(-1)[at_ring] = s["scores"][wr, rr - s["prefix"][wr]]
    return _pack_plain(s["K_pool"], s["V_pool"], s["table"], s["prefix"], s["K_ring"], s["V_ring"], s["score_ring"], s["tokens"], page)


def _exact_move(case, seed):
    counts, start, K, V, tokens, scores = _move_inputs(case, seed)
    return [K.double(), V.double(), start, tokens, scores.double()]


def _work_move(case):
    n = case["seqs"] * case["layers"] * H
    rows = sum(_lengths(case, n)) + n * min(case["tokens"], case["window"])
    return {"bytes": 4 * rows * case["dim"] * 4, "flops": 0}


# --------------------------------------------------------------------------------------------------------------- attend

def _attend_inputs(case, seed):
    """Prefixes of the groups in pages, the rows that each member has appended since, and the new token's queries."""
    g, m, L, D, page, steps = (case[k] for k in ("groups", "members", "layers", "dim", "page", "steps"))
    counts = _lengths(case, g * L * H)
    width = -(-max(counts) // page) + -(-steps // page) + 2
    table, used = _tables(counts, page, width, _gen(seed, 0))
    n_pages = used + g * m * L * H * (max(0, steps - case["window"]) // page + 2)
    K_pool, V_pool = (_normal(_gen(seed, 1 + i), n_pages, page, D) for i in range(2))
    K_new, V_new = (_normal(_gen(seed, 3 + i), steps, L, g * m, H, D) for i in range(2))
    Q = _normal(_gen(seed, 5), L, g * m, H * case["per_kv"], D) * 2
    return counts, width, table, used, K_pool, V_pool, K_new, V_new, Q


def _prepare_attend(case, seed):
    g, m, L, D = (case[k] for k in ("groups", "members", "layers", "dim"))
    counts, width, table, used, K_pool, V_pool, K_new, V_new, Q = _attend_inputs(case, seed)
    s = {"Q": Q}
    if own:
        s["session"] = session = _Session(L, D, max(64, g * m))
        for l in range(L):
            session.ctx.set_weights(l, torch.zeros(H, 64, dtype=torch.bfloat16, device="cuda"), None)
        session.open_cache(g * m, case, K_pool, V_pool, width)
        cache = session.cache
        full_table = torch.zeros(g, m, L * H, width, dtype=torch.int32, device="cuda")
        full_table[:, 0] = table.view(g, L * H, width)
        prefix = torch.zeros(g, m, L * H, dtype=torch.int32, device="cuda")
        prefix[:, 0] = _int(counts).view(g, L * H)
        cache.import_prefix(prefix.view(-1), full_table.view(-1, width), used)
        cache.fork([b // m * m for b in range(g * m) if b % m], [b for b in range(g * m) if b % m])
        hidden = torch.zeros(L, g * m, 64, dtype=torch.bfloat16, device="cuda")
        for t in range(case["steps"]):
            cache.decode_step(0, L, hidden, K_new[t], V_new[t], MINUS_INF)
        cache.share([list(range(a * m, (a + 1) * m)) for a in range(g)], H * case["per_kv"])
        s["O"] = torch.empty_like(Q)
        s["keep"] = (K_pool, V_pool)
        return s
    s.update(K_pool=K_pool, V_pool=V_pool, table=table[:, :-(-max(counts) // case["page"])].long(), prefix=_int(counts, torch.int64),
             K_new=K_new, V_new=V_new)
    return s


def _run_attend(s):
    case = s["case"]
    g, m, L, D, G = (case[k] for k in ("groups", "members", "layers", "dim", "per_kv"))
    if own:
        return s["session"].cache.attention_shared(0, L, s["Q"], out=s["O"])
    Q = s["Q"].float().view(L, g, m, H, G, D).permute(1, 0, 3, 2, 4, 5)                    # [g, L, H, m, G, D]
    K, V = (s[k][s["table"]].float().view(g, L, H, -1, D) for k in ("K_pool", "V_pool"))
    Kn, Vn = (s[k].float().view(-1, L, g, m, H, D).permute(2, 1, 4, 3, 0, 5) for k in ("K_new", "V_new"))
    shared = (Q.reshape(g, L, H, m * G, D) @ K.transpose(-1, -2)).view(g, L, H, m, G, -1)
    absent = torch.arange(shared.shape[-1], device="cuda") >= s["prefix"].view(g, L, H, 1, 1, 1)
    logits = torch.cat([shared.masked_fill(absent, MINUS_INF), Q @ Kn.transpose(-1, -2)], -1) * D ** -0.5
    p = (logits - logits.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    n = shared.shape[-1]
    O = (p[..., :n].reshape(g, L, H, m * G, n) @ V).view(g, L, H, m, G, D) + p[..., n:] @ Vn
    return O.permute(1, 0, 3, 2, 4, 5).reshape(L, g * m, H * G, D).bfloat16()


def _exact_attend(case, seed):
    g, m, L, D, G = (case[k] for k in ("groups", "members", "layers", "dim", "per_kv"))
    counts, width, table, used, K_pool, V_pool, K_new, V_new, Q = _attend_inputs(case, seed)
    O = torch.empty(L, g * m, H * G, D, dtype=torch.float64, device="cuda")
    for a in range(g):
        for l in range(L):
            for h in range(H):
                i = (a * L + l) * H + h
                pages = table[i, :-(-counts[i] // case["page"])].long()
                K, V = (pool[pages].reshape(-1, D)[:counts[i]].double() for pool in (K_pool, V_pool))
                for b in range(a * m, (a + 1) * m):
                    q = Q[l, b, h * G:(h + 1) * G].double()
                    x = torch.cat([K @ q.t(), K_new[:, l, b, h].double() @ q.t()]) / math.sqrt(D)
                    p = torch.softmax(x, 0)
                    O[l, b, h * G:(h + 1) * G] = p[:counts[i]].t() @ V + p[counts[i]:].t() @ V_new[:, l, b, h].double()
    return O


def _work_attend(case):
    g, m, L, D, G = (case[k] for k in ("groups", "members", "layers", "dim", "per_kv"))
    rows = sum(_lengths(case, g * L * H))
    mine = g * m * L * H * case["steps"]
    return {"bytes": (rows + mine) * D * 4 + 2 * g * m * L * H * G * D * 2, "flops": 4 * D * G * (rows * m + mine)}
