"""Timed cases of serving drafts and branches over the paged 8-bit K/V cache, and of rotations by positions of several
axes, with plain forms of each.

Three operators, six kinds of case:

  "tree"     attention of a tree of drafted tokens over the cache: a row sees the tokens before the drafts (through the
             layer's window and sinks) and the drafted tokens that its mask names; O and LSE
  "draft"    drafted tokens into the cache: masks and positions of the tree from each token's parent, then K (and Q)
             rotated by those positions and the codes written
  "image"    prompts of text and images into the cache, rotated by positions of several axes
  "rotate"   the same rotation in training: q and k forward, and their gradients back
  "compact"  kept tokens of every sequence move together: the accepted ones of a tree, or what an eviction keeps
  "pages"    one step of branching sequences: rows of the page table become other rows, pages for the new tokens, copies
             of the shared pages that are about to be written

`own` false: elementary torch operations in 32 bits.  `own` true: this package's entry points.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0
MIN_EXP, MAX_EXP = -100, 120   # range of a scale's exponent
NO_WINDOW = 2 ** 31 - 1


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _tree(seqs, nodes, held, page, heads_q, heads_kv, dim, window=NO_WINDOW, sinks=0, shape=0):
    return {"kind": "tree", "seqs": seqs, "new": nodes, "held": held, "page": page, "heads_q": heads_q,
            "heads_kv": heads_kv, "dim": dim, "window": window, "sinks": sinks, "shape": shape}


def _draft(seqs, nodes, held, page, heads_q, heads_kv, dim, rot, interleaved=False, shape=0):
    return {"kind": "draft", "seqs": seqs, "new": nodes, "held": held, "page": page, "heads_q": heads_q,
            "heads_kv": heads_kv, "dim": dim, "rot": rot, "axes": 1, "order": "runs", "interleaved": interleaved,
            "k_out": False, "shape": shape}


def _image(seqs, new, held, page, heads_q, heads_kv, dim, rot, axes, order, interleaved=False, k_out=True, shape=0):
    return {"kind": "image", "seqs": seqs, "new": new, "held": held, "page": page, "heads_q": heads_q,
            "heads_kv": heads_kv, "dim": dim, "rot": rot, "axes": axes, "order": order, "interleaved": interleaved,
            "k_out": k_out, "shape": shape}


def _rotate_case(tokens, heads_q, heads_kv, dim, rot, axes, order, interleaved=False, shape=0):
    return {"kind": "rotate", "tokens": tokens, "heads_q": heads_q, "heads_kv": heads_kv, "dim": dim, "rot": rot,
            "axes": axes, "order": order, "interleaved": interleaved, "shape": shape}


def _compact(seqs, new, held, page, heads_kv, dim, keep, fresh, shape=0):
    """keep: share of the `new` last tokens that stay; fresh: into other pages than they are in."""
    return {"kind": "compact", "seqs": seqs, "new": new, "held": held, "page": page, "heads_kv": heads_kv, "dim": dim,
            "keep": keep, "fresh": fresh, "shape": shape}


def _pages(seqs, branch, new, held, page, heads_kv, dim, layers, shape=0):
    """Groups of `branch` rows that all go on from their group's first."""
    return {"kind": "pages", "seqs": seqs, "branch": branch, "new": new, "held": held, "page": page,
            "heads_kv": heads_kv, "dim": dim, "layers": layers, "shape": shape}


def listed():
    return [
        # a small model's drafts of one user: the smallest call, launches count
        dict(_tree(1, 16, 1000, 16, 4, 4, 64), name="tree 1x16 over 1k d64"),
        # an ordinary batch that verifies a tree for every sequence
        dict(_tree(32, 24, 4096, 64, 32, 8, 128), name="tree 32x24 over 4k"),
        # wide trees over long contexts
        dict(_tree(8, 64, 32768, 128, 32, 8, 128), name="tree 8x64 over 32k"),
        # a window layer; trees of more than 64 tokens
        dict(_tree(5, 100, 6000, 16, 12, 2, 64, window=1024, sinks=4), name="tree 5x100 w1024 d64"),
        # the ordinary batch's drafts on their way into the cache
        dict(_draft(32, 24, 4096, 64, 32, 8, 128, 128), name="draft 32x24"),
        # prompts of text and images into empty pages; rotated K kept for the prompt's own attention
        dict(_image(4, 2500, 0, 32, 32, 8, 128, 128, 3, "runs"), name="append images 4x2500"),
        # an odd batch of a small image model in training, two axes, half of each head rotated
        dict(_rotate_case(1999, 6, 2, 64, 32, 2, "turns", interleaved=True), name="rotate 2k d64"),
        # video training: three axes, every head of a large layer
        dict(_rotate_case(32768, 32, 8, 128, 128, 3, "turns"), name="rotate 32k"),
        # accepted tokens of the ordinary batch's trees
        dict(_compact(32, 24, 4096, 64, 8, 128, 0.2, False), name="keep accepted 32x24"),
        # half of every context evicted, the rest into fresh pages
        dict(_compact(16, 8192, 0, 64, 8, 128, 0.5, True), name="evict half of 16x8k"),
        # beam search of a small model
        dict(_pages(8, 4, 1, 1000, 16, 4, 64, 1), name="fork 2x4 beams"),
        # several samples of every prompt, all layers' caches on one page table
        dict(_pages(64, 4, 1, 4096, 128, 8, 128, 4), name="fork 16x4 samples"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(["tree", "tree", "tree", "draft", "image", "rotate", "compact", "compact", "pages"])
    dim = rng.choice([64, 128])
    heads_kv = rng.choice([1, 2, 3, 4, 8])
    heads_q = heads_kv * rng.choice([1, 2, 4, 5, 8])
    page = rng.choice([16, 32, 64, 128])
    rot = rng.choice([dim // 4, dim // 2, dim])
    axes = rng.choice([1, 2, 3, 4])
    order = rng.choice(["runs", "turns"])
    shape = rng.randrange(1 << 20)
    if kind == "rotate":
        return _rotate_case(log(1, 16384), heads_q, heads_kv, dim, rot, axes, order, rng.random() < 0.5, shape)
    seqs = log(1, 64)
    if kind == "tree":
        held, nodes = log(1, 200000 // seqs), log(1, min(300, max(1, 1024 // seqs)))
        # no more work than the largest listed case
        nodes = max(1, min(nodes, 2 * 10 ** 11 // (4 * seqs * held * heads_q * dim)))
        return _tree(seqs, nodes, held, page, heads_q, heads_kv, dim, rng.choice([NO_WINDOW, log(1, held)]),
                     rng.choice([0, 4, 20]), shape)
    if kind == "draft":
        return _draft(seqs, log(1, min(300, max(1, 1024 // seqs))), log(1, 8192), page, heads_q, heads_kv, dim, rot,
                      rng.random() < 0.5, shape)
    if kind == "image":
        return _image(seqs, log(1, 8192 // seqs), rng.choice([0, log(1, 4096)]), page, heads_q, heads_kv, dim, rot, axes,
                      order, rng.random() < 0.5, rng.random() < 0.5, shape)
    if kind == "compact":
        fresh = rng.random() < 0.5
        return _compact(seqs, log(1, 65536 // seqs if fresh else 300), 0 if fresh else log(1, 4096), page, heads_kv, dim,
                        round(rng.uniform(0.05, 1.0), 3), fresh, shape)
    branch = rng.choice([1, 2, 3, 4, 8])
    return _pages(branch * log(1, 64 // branch), branch, log(1, 64), log(1, 8192), page, heads_kv, dim,
                  rng.choice([1, 2, 4]), shape)


# ---------------------------------------------------------------------------
# lengths, trees, positions (host)
# ---------------------------------------------------------------------------

def _lens(case):
    """Tokens per sequence before (`held`) and on top (`new`): ragged where there are several sequences (a quarter to
    all of the case's size; now and then none)."""
    rng = np.random.default_rng(case["shape"] + 17)
    s = case["seqs"]
    if s == 1:
        return np.array([case["held"]]), np.array([case["new"]])
    held = (case["held"] * rng.uniform(0.25, 1.0, s)).astype(np.int64)
    new = np.full(s, case["new"], dtype=np.int64)
    if case["new"] > 1:
        new = np.maximum(1, (case["new"] * rng.uniform(0.25, 1.0, s)).astype(np.int64))
        if s > 2:
            new[rng.integers(0, s)] = 0
    return held, new


def _parents(case, new):
    """Every drafted token's parent among its sequence's drafted tokens: one of the eight before it, or none (-1)."""
    rng = np.random.default_rng(case["shape"] + 23)
    out = [rng.integers(max(-1, j - 8), j) for n in new for j in range(int(n))]
    return np.array(out, dtype=np.int32)


def _tree_of(new, parents, words):
    """(own and ancestors' bits [total, words] as int64, depth [total])"""
    bits = np.zeros((len(parents), words), dtype=np.uint64)
    depth = np.zeros(len(parents), dtype=np.int64)
    at = 0
    for n in new:
        for j in range(int(n)):
            p = int(parents[at + j])
            if p >= 0:
                bits[at + j] = bits[at + p]
                depth[at + j] = depth[at + p] + 1
            bits[at + j, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        at += int(n)
    return bits.view(np.int64), depth


def _axis_of_pairs(case):
    """Axis of every pair: one run of pairs per axis, or the axes in turn."""
    pairs, axes = case["rot"] // 2, case["axes"]
    i = np.arange(pairs)
    return (i * axes // pairs if case["order"] == "runs" else i % axes).astype(np.uint8)


def _grid_positions(total, axes, rng):
    """Positions [axes, total] of text (every axis the same) and images (frame, row, column, then their sum) by turns."""
    out = np.zeros((4, total), dtype=np.int32)
    at = base = 0
    while at < total:
        n = min(total - at, int(rng.integers(20, 200)))
        out[:, at:at + n] = base + np.arange(n)
        at, base = at + n, base + n
        h, w = int(rng.integers(4, 40)), int(rng.integers(4, 40))
        n = min(total - at, h * w)
        i = np.arange(n)
        out[:, at:at + n] = base + np.stack([0 * i, i // w, i % w, i // w + i % w])
        at, base = at + n, base + h + w
    return {1: out[3:], 2: out[1:3], 3: out[:3], 4: out}[axes]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _randn(shape, g, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _cuda(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(dtype))).cuda()


def _page_exponent(amax):
    """Exponent of a page's scale: the smallest e with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax / E4M3_MAX)                # amax / 448 = m 2^e, m in [0.5, 1)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.where(amax > 0, e, torch.full_like(e, MIN_EXP)).clamp(MIN_EXP, MAX_EXP)


def _encode(x):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)


def _filled(pages, hkv, page, d, g):
    """Codes and scales of unit normal values whose size varies from page to page, as appends leave them."""
    codes = torch.empty((pages, hkv, page, d), dtype=torch.uint8, device="cuda")
    scales = torch.empty((pages, hkv), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 27) // (hkv * page * d))
    for a in range(0, pages, step):
        n = min(step, pages - a)
        val = torch.randn((n, hkv, page, d), generator=g, device="cuda")
        val *= torch.exp(0.5 * torch.randn((n, hkv, 1, 1), generator=g, device="cuda"))
        sc = torch.ldexp(torch.ones((), device="cuda"), _page_exponent(val.abs().amax((2, 3))))
        codes[a:a + step] = _encode(val / sc[:, :, None, None])
        scales[a:a + step] = sc
    return codes, scales


def _tables(case, total, spare=3):
    """Pages of every sequence's `total` tokens, in random order among all: table, number of pages, pages in no row."""
    page = case["page"]
    per = -(-np.asarray(total) // page)
    width, pages = max(1, int(per.max())), int(per.sum()) + spare
    order = np.random.default_rng(case["shape"] + 5).permutation(pages)
    table = np.full((len(per), width), -1, dtype=np.int64)
    at = 0
    for i, n in enumerate(per):
        table[i, :n] = order[at:at + int(n)]
        at += int(n)
    return table, pages, order[at:]


def _touch(table, page, first, count):
    """Pages that tokens first .. first + count - 1 of every sequence reach, and the first slot of each that they take."""
    touched, slot = [], []
    for i in range(len(first)):
        if count[i]:
            for p in range(int(first[i]) // page, int(first[i] + count[i] - 1) // page + 1):
                touched.append(int(table[i, p]))
                slot.append(max(0, int(first[i]) - p * page))
    return _cuda(touched, np.int64), _cuda(slot, np.int64)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"tree": _prepare_tree, "draft": _prepare_new, "image": _prepare_new, "rotate": _prepare_rotate,
            "compact": _prepare_compact, "pages": _prepare_pages}[case["kind"]](case, g)


def _cos_sin(rows, rot):
    f = 10000.0 ** (-np.arange(rot // 2) * 2.0 / rot)
    angle = np.arange(rows)[:, None] * f[None]
    return _cuda(np.concatenate([np.cos(angle), np.sin(angle)], 1), np.float32)


def _with_cache(s, pages, table, lens, g):
    case = s["case"]
    for x in ("k", "v"):
        s[x + "_codes"], s[x + "_scale"] = _filled(pages, case["heads_kv"], case["page"], case["dim"], g)
    s["table"], s["lens"] = _cuda(table), _cuda(lens)
    return s


def _new_tokens(case):
    """A state with the new tokens' places."""
    held, new = _lens(case)
    table, pages, _ = _tables(case, held + new)
    s = {"case": case, "scale": 1.0 / math.sqrt(case["dim"]), "total_new": int(new.sum()), "max_new": int(new.max()),
         "cu": _cuda(np.concatenate([[0], np.cumsum(new)]))}
    return s, held, new, table, pages


def _prepare_tree(case, g):
    s, held, new, table, pages = _new_tokens(case)
    hq, d, t = case["heads_q"], case["dim"], s["total_new"]
    s["words"] = -(-int(new.max()) // 64)
    bits, depth = _tree_of(new, _parents(case, new), s["words"])
    s["mask"] = torch.from_numpy(bits).cuda()
    s["positions"] = _cuda(np.repeat(held, new) + depth)
    s["q"] = _randn((t, hq, d), g)
    s["o"] = torch.empty((t, hq, d), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.empty((hq, t), dtype=torch.float32, device="cuda")
    return _with_cache(s, pages, table, held + new, g)


def _prepare_new(case, g):
    s, held, new, table, pages = _new_tokens(case)
    hq, hkv, d, t = case["heads_q"], case["heads_kv"], case["dim"], s["total_new"]
    if case["kind"] == "draft":
        s["words"] = -(-int(new.max()) // 64)
        s["parents"] = _cuda(_parents(case, new))
        s["mask"] = torch.empty((t, s["words"]), dtype=torch.int64, device="cuda")
        s["positions"] = torch.empty((1, t), dtype=torch.int32, device="cuda")
    else:
        rng = np.random.default_rng(case["shape"] + 31)
        s["positions"] = _cuda(np.concatenate([_grid_positions(int(n), case["axes"], rng) + int(a) for a, n in zip(held, new)], 1))
    s["axis"] = _axis_of_pairs(case)
    s["cos_sin"] = _cos_sin(int((held + new).max()) + 2, case["rot"])
    qkv = _randn((t, hq + 2 * hkv, d), g)              # the fused projection's rows
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    s["q_out"] = torch.empty((t, hq, d), dtype=torch.bfloat16, device="cuda")
    s["k_out"] = torch.empty((t, hkv, d), dtype=torch.bfloat16, device="cuda") if case["k_out"] else None
    s["touched"], s["first"] = _touch(table, case["page"], held, new)
    return _with_cache(s, pages, table, held + new, g)


def _prepare_rotate(case, g):
    t, hq, hkv, d = case["tokens"], case["heads_q"], case["heads_kv"], case["dim"]
    rng = np.random.default_rng(case["shape"] + 31)
    qkv = _randn((t, hq + 2 * hkv, d), g)
    s = {"case": case, "positions": _cuda(_grid_positions(t, case["axes"], rng)), "axis": _axis_of_pairs(case),
         "cos_sin": _cos_sin(t + 100, case["rot"]), "q": qkv[:, :hq], "k": qkv[:, hq:hq + hkv],
         # gradients as the attention's backward leaves them: dK in fp32, summed over shards
         "d_q": _randn((t, hq, d), g), "d_k": _randn((t, hkv, d), g, torch.float32)}
    for x, h in (("q", hq), ("k", hkv)):
        s[x + "_out"] = torch.empty((t, h, d), dtype=torch.bfloat16, device="cuda")
    grad = torch.empty((t, hq + 2 * hkv, d), dtype=torch.bfloat16, device="cuda")   # the fused projection's gradient
    s["q_grad"], s["k_grad"] = grad[:, :hq], grad[:, hq:hq + hkv]
    return s


def _kept(case, held, new):
    """Positions that stay, per sequence: of the `new` last tokens a share, ascending."""
    rng = np.random.default_rng(case["shape"] + 41)
    return [int(a) + np.sort(rng.permutation(int(n))[:min(int(n), max(1, int(round(case["keep"] * int(n)))))])
            for a, n in zip(held, new)]


def _prepare_compact(case, g):
    s, held, new, table, pages = _new_tokens(case)
    kept = _kept(case, held, new)
    count = np.array([len(k) for k in kept])
    target = table
    if case["fresh"]:
        per = -(-count // case["page"])
        target = np.full_like(table, -1)
        at = pages
        for i, n in enumerate(per):
            target[i, :n] = at + np.arange(n)
            at += int(n)
        pages = at
        s["dst_table"] = _cuda(target)
    s["keep"], s["cu_keep"] = _cuda(np.concatenate(kept)), _cuda(np.concatenate([[0], np.cumsum(count)]))
    s["start"] = _cuda(held)
    s["new_lens"] = torch.empty(case["seqs"], dtype=torch.int32, device="cuda")
    s["touched"], s["first"] = _touch(target, case["page"], held, count)
    return _with_cache(s, pages, table, held + new, g)


def _prepare_pages(case, g):
    held, new = _lens(case)
    seqs, page, branch = case["seqs"], case["page"], case["branch"]
    lead = np.arange(seqs) // branch * branch
    committed = np.where(lead == np.arange(seqs), held, 0)    # the groups' first rows alone hold something yet
    own_pages, pages, _ = _tables(case, committed, spare=0)
    width = max(own_pages.shape[1], int((-(-(held[lead] + new) // page)).max()))
    table = np.full((seqs, width), -1, dtype=np.int64)
    table[:, :own_pages.shape[1]] = own_pages
    room = int((-(-new // page) + 2).sum())
    pages += room
    # rows over the whole range of pages, so that free ones lie between those in use
    place = np.random.default_rng(case["shape"] + 6).permutation(pages)
    table = np.where(table >= 0, place[np.maximum(table, 0)], -1)
    refs = np.bincount(table[table >= 0], minlength=pages)
    s = {"case": case, "source": _cuda(lead), "refs": _cuda(refs), "committed": _cuda(committed),
         "cu": _cuda(np.concatenate([[0], np.cumsum(new)])), "new": _cuda(new), "total_new": int(new.sum()),
         "table": _cuda(table), "lens": _cuda(committed), "reach": int(-(-int(new.max()) // page)) + 1, "layers": [],
         "pairs": torch.empty((seqs, 2), dtype=torch.int32, device="cuda"),
         "missing": torch.empty(1, dtype=torch.int32, device="cuda")}
    for _ in range(case["layers"]):
        layer = {}
        for x in ("k", "v"):
            layer[x + "_codes"], layer[x + "_scale"] = _filled(pages, case["heads_kv"], page, case["dim"], g)
        s["layers"].append(layer)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return {"tree": _run_tree, "draft": _run_new, "image": _run_new, "rotate": _run_rotate, "compact": _run_compact,
            "pages": _run_pages}[s["case"]["kind"]](s)


def _own(s):
    from paper_2606_30460_amd import _lib as L
    c = s["case"]
    if "ready" not in s:    # the handles and workspaces that a program keeps
        s["ready"] = True
        if "cos_sin" in s:
            s["rotation"] = L.Rotation(s["cos_sin"], s["axis"], c["interleaved"])
        if "k_codes" in s:
            s["cache"] = L.KVCache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["table"], s["lens"])
        size = 0
        if c["kind"] == "tree":
            size = L.cache_tree_attn_workspace(s["cache"], c["heads_q"], s["total_new"])
        if c["kind"] == "pages":
            s["caches"] = [L.KVCache(y["k_codes"], y["v_codes"], y["k_scale"], y["v_scale"], s["table"], s["lens"])
                           for y in s["layers"]]
            size = L.pages_reserve_workspace(s["caches"][0], s["total_new"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return L


def _cache_out(s):
    return [s["k_codes"].view(torch.float8_e4m3fn), s["k_scale"], s["v_codes"].view(torch.float8_e4m3fn), s["v_scale"]]


def _run_tree(s):
    if own:
        L, c = _own(s), s["case"]
        L.cache_tree_attn(s["cache"], c["heads_q"], s["scale"], s["q"], s["cu"], s["mask"], s["positions"], s["o"], s["lse"],
                          s["workspace"], window=c["window"], sinks=c["sinks"])
        return [s["o"], s["lse"]]
    return _plain_tree(s)


def _run_new(s):
    if own:
        L = _own(s)
        drafted = s["case"]["kind"] == "draft"
        if drafted:
            L.tree_masks(s["lens"], s["cu"], s["parents"], s["mask"], s["positions"])
        L.cache_append_at(s["cache"], s["k"], s["v"], s["cu"], s["rotation"], s["positions"], k_out=s["k_out"], q=s["q"],
                          q_out=s["q_out"])
        out = [s["q_out"]] + _cache_out(s) + ([s["k_out"]] if s["k_out"] is not None else [])
        return out + ([s["mask"], s["positions"]] if drafted else [])
    return _plain_new(s)


def _run_rotate(s):
    if own:
        L = _own(s)
        L.rotate(s["rotation"], s["positions"], s["q"], s["q_out"], s["k"], s["k_out"])
        L.rotate(s["rotation"], s["positions"], s["d_q"], s["q_grad"], s["d_k"], s["k_grad"], inverse=True)
        return [s["q_out"], s["k_out"], s["q_grad"], s["k_grad"]]
    return _plain_rotate(s)


def _run_compact(s):
    if own:
        L = _own(s)
        L.cache_compact(s["cache"], s["keep"], s["cu_keep"], first=s["start"], dst_table=s.get("dst_table"),
                        new_lens=s["new_lens"])
        return _cache_out(s) + [s["new_lens"]]
    return _plain_compact(s)


def _pages_out(s):
    out = [s["table"], s["committed"], s["lens"], s["refs"], s["pairs"], s["missing"]]
    for y in s["layers"]:
        out += [y["k_codes"].view(torch.float8_e4m3fn), y["k_scale"], y["v_codes"].view(torch.float8_e4m3fn), y["v_scale"]]
    return out


def _run_pages(s):
    if own:
        L = _own(s)
        L.pages_fork(s["caches"][0], s["refs"], s["source"], seq_lens=s["committed"])
        torch.add(s["committed"], s["new"], out=s["lens"])
        L.pages_reserve(s["caches"][0], s["refs"], s["cu"], s["total_new"], s["pairs"], s["missing"], s["workspace"])
        for cache in s["caches"]:
            L.cache_copy_pages(cache, s["pairs"])
        return _pages_out(s)
    return _plain_pages(s)


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _places(s):
    """Sequence of every new token and its number within it (tensors)."""
    t = torch.arange(s["total_new"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu"], t, right=True) - 1
    return seq, t.long() - s["cu"].long()[seq]


def _decoded(codes, scales, table):
    """Values [seqs, Hkv, tokens, d] of the pages in `table`."""
    seqs, width = table.shape
    _, hkv, page, d = codes.shape
    at = table.clamp(min=0)
    val = codes[at].view(torch.float8_e4m3fn).float() * scales[at][..., None, None]
    return val.permute(0, 2, 1, 3, 4).reshape(seqs, hkv, width * page, d)


def _plain_tree(s):
    case = s["case"]
    hq, hkv, d, seqs, most = case["heads_q"], case["heads_kv"], case["dim"], case["seqs"], s["max_new"]
    grp, table = hq // hkv, s["table"].long()
    k, v = (_decoded(s[x + "_codes"], s[x + "_scale"], table) for x in "kv")
    cu, lens = s["cu"].long(), s["lens"].long()
    base = lens - cu.diff()
    row = (cu[:-1, None] + torch.arange(most, device="cuda")).clamp(max=s["total_new"] - 1)               # [seqs, T]
    pos = s["positions"].long()[row]
    j = torch.arange(k.shape[2], device="cuda")
    node = j - base[:, None]                                                                               # [seqs, tokens]
    at = node.clamp(min=0, max=most - 1)
    place = torch.where(node < 0, j, pos.gather(1, at))                                                    # a token's position
    bit = (s["mask"][row].gather(2, (at // 64)[:, None].expand(seqs, most, -1)) >> (at % 64)[:, None]) & 1
    dist = pos[:, :, None] - place[:, None]
    ok = ((node < 0)[:, None] | (bit == 1)) & ((dist < case["window"]) | (place < case["sinks"])[:, None])
    ok &= (j < lens[:, None])[:, None]
    q = s["q"].float()[row].view(seqs, most, hkv, grp, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, grp * most, d)
    sc = (q @ k.transpose(2, 3)).view(seqs, hkv, grp, most, -1) * s["scale"]
    sc = sc.masked_fill(~ok[:, None, None], -math.inf)
    top = sc.amax(-1)
    p = (sc - top.masked_fill(top == -math.inf, 0.0)[..., None]).exp()
    den = p.sum(-1)
    o = (p.view(seqs, hkv, grp * most, -1) @ v).view(seqs, hkv, grp, most, d) / den.clamp(min=1e-30)[..., None]
    lse = top + den.log()
    seq, t = _places(s)
    o = o.permute(0, 3, 1, 2, 4).reshape(seqs, most, hq, d)[seq, t]
    lse = lse.permute(0, 3, 1, 2).reshape(seqs, most, hq)[seq, t]
    return [o.to(torch.bfloat16), lse.t().contiguous()]


def _turn(x, cos, sin, rot, interleaved):
    """Pairs of the first `rot` values of every head's row by cos, sin [tokens, rot / 2]."""
    x = x.float()
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _rows_of(s, positions):
    """cos and sin [tokens, rot / 2] of every token's pairs, each from the row of its axis."""
    half = s["case"]["rot"] // 2
    pair = torch.arange(half, device="cuda")
    row = positions.long()[torch.from_numpy(s["axis"].astype(np.int64)).cuda()].t()                        # [tokens, pairs]
    return s["cos_sin"][row, pair], s["cos_sin"][row, half + pair]


def _plain_masks(s):
    """Bits and positions of the drafted tokens: chains of parents, twice as far with every turn."""
    seq, me = _places(s)
    cu = s["cu"].long()
    base = s["lens"].long() - cu.diff()
    parents = s["parents"].long()
    words = torch.arange(s["words"], device="cuda")
    mask = torch.where(me[:, None] // 64 == words, (torch.ones_like(me) << (me % 64))[:, None], 0)
    above = torch.where(parents >= 0, cu[seq] + parents, -1)   # the first token of the chain that is not counted yet
    depth = torch.ones_like(me)
    for _ in range(s["max_new"].bit_length()):
        live, at = above >= 0, above.clamp(min=0)
        mask = mask | torch.where(live[:, None], mask[at], 0)
        depth = depth + torch.where(live, depth[at], 0)
        above = torch.where(live, above[at], -1)
    return mask, (base[seq] + depth - 1).int()[None]


def _plain_write(s, values, name, at, slot):
    """Values [tokens, Hkv, d] into the pages `at`, places `slot`: scales raised where they have to be, older codes of a page
    encoded again."""
    codes, scales = s[name + "_codes"], s[name + "_scale"]
    page, touched, first = codes.shape[2], s["touched"], s["first"]
    amax = torch.zeros_like(scales).index_reduce_(0, at, values.abs().amax(-1), "amax")[touched]
    need = torch.ldexp(torch.ones_like(amax), _page_exponent(amax))
    before = scales[touched]
    after = torch.where(first[:, None] > 0, torch.maximum(need, before), need)
    again = _encode(codes[touched].view(torch.float8_e4m3fn).float() * (before / after)[:, :, None, None])
    old = (torch.arange(page, device="cuda")[None] < first[:, None])[:, None, :, None]
    codes[touched] = torch.where(old, again, codes[touched])
    scales[touched] = after
    codes[at, :, slot] = _encode(values / scales[at][..., None])


def _plain_new(s):
    case = s["case"]
    page, rot, il = case["page"], case["rot"], case["interleaved"]
    drafted = case["kind"] == "draft"
    seq, me = _places(s)
    place = (s["lens"].long() - s["cu"].long().diff())[seq] + me
    mask, positions = _plain_masks(s) if drafted else (None, s["positions"])
    cos, sin = _rows_of(s, positions)
    q, k = (_turn(s[x], cos, sin, rot, il) for x in "qk")
    at, slot = s["table"].long()[seq, place // page], place % page
    _plain_write(s, k, "k", at, slot)
    _plain_write(s, s["v"].float(), "v", at, slot)
    out = [q.to(torch.bfloat16)] + _cache_out(s) + ([k.to(torch.bfloat16)] if s["k_out"] is not None else [])
    return out + ([mask, positions] if drafted else [])


def _plain_rotate(s):
    rot, il = s["case"]["rot"], s["case"]["interleaved"]
    cos, sin = _rows_of(s, s["positions"])
    out = [_turn(s["q"], cos, sin, rot, il), _turn(s["k"], cos, sin, rot, il), _turn(s["d_q"], cos, -sin, rot, il),
           _turn(s["d_k"], cos, -sin, rot, il)]
    return [x.to(torch.bfloat16) for x in out]


def _plain_compact(s):
    page = s["case"]["page"]
    i = torch.arange(s["keep"].numel(), device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu_keep"], i, right=True) - 1
    place = s["start"].long()[seq] + i.long() - s["cu_keep"].long()[seq]
    source = s["keep"].long()
    table = s["table"].long()
    target = s["dst_table"].long() if "dst_table" in s else table
    src, at = table[seq, source // page], target[seq, place // page]
    values = [s[x + "_codes"][src, :, source % page].view(torch.float8_e4m3fn).float() * s[x + "_scale"][src][..., None]
              for x in "kv"]
    _plain_write(s, values[0], "k", at, place % page)
    _plain_write(s, values[1], "v", at, place % page)
    s["new_lens"].copy_(s["start"] + s["cu_keep"].diff())
    return _cache_out(s) + [s["new_lens"]]


def _plain_pages(s):
    case = s["case"]
    page, seqs = case["page"], case["seqs"]
    table, refs = s["table"].long(), s["refs"].long()
    pages, width = refs.numel(), table.shape[1]
    one = torch.ones(1, dtype=torch.int64, device="cuda")

    def count(t):     # entries per page
        return torch.zeros(pages + 1, dtype=torch.int64, device="cuda").index_add_(0, (t + (t < 0) * (pages + 1)).reshape(-1),
                                                                                   one.expand(t.numel()))[:pages]

    # rows become other rows, pages behind their lengths are given back
    src = s["source"].long()
    lens = s["committed"].long()[src]
    column = torch.arange(width, device="cuda")
    forked = torch.where(column < -(-lens[:, None] // page), table[src], -1)
    refs = refs + count(forked) - count(table)
    busy = refs.argmax()
    s["committed"].copy_(lens)
    s["lens"].copy_(lens + s["new"])
    # pages for the new tokens: [seqs, reach]
    new = s["new"].long()
    a = lens[:, None] // page + torch.arange(s["reach"], device="cuda")
    write = (a * page < (lens + new)[:, None]) & (new[:, None] > 0)
    ac = a.clamp(max=width - 1)
    has = forked.gather(1, ac)
    held = write & (has >= 0)
    hc = has.clamp(min=0)
    writers = torch.zeros(pages, dtype=torch.int64, device="cuda").index_add_(0, hc.reshape(-1), held.long().reshape(-1))
    row = torch.arange(seqs, device="cuda")[:, None].expand_as(a)
    last = torch.full((pages,), -1, dtype=torch.int64, device="cuda").index_reduce_(
        0, hc.reshape(-1), torch.where(held, row, torch.full_like(row, -1)).reshape(-1), "amax")
    keeps = held & (refs[hc] == writers[hc]) & (last[hc] == row)
    need = write & ~keeps
    nth = need.reshape(-1).long().cumsum(0)
    free = (refs == 0).long().cumsum(0)
    missing = (nth[-1] - free[-1]).clamp(min=0)
    fine = need & (missing == 0)
    got = torch.searchsorted(free, nth).view_as(a).clamp(max=pages - 1)
    wide = torch.cat([forked, forked[:, :1]], 1)      # (a column for the places that are not written)
    s["table"].copy_(wide.scatter(1, torch.where(write, ac, width), torch.where(fine, got, has))[:, :width])
    refs = refs - torch.zeros_like(refs).index_add_(0, hc.reshape(-1), (fine & held).long().reshape(-1))
    refs = refs + torch.zeros_like(refs).index_add_(0, got.reshape(-1), fine.long().reshape(-1))
    s["refs"].copy_(refs)
    copied = fine[:, 0] & held[:, 0] & (lens % page > 0)
    pairs = torch.where(copied[:, None], torch.stack([has[:, 0], got[:, 0]], 1), -1)
    s["pairs"].copy_(pairs)
    s["missing"].copy_(missing)
    # copies; a pair that is none copies a page in use onto itself
    of, to = (torch.where(copied, pairs[:, i], busy) for i in (0, 1))
    for y in s["layers"]:
        for t in y.values():
            t[to] = t[of]
    return _pages_out(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    hkv, d = case["heads_kv"], case["dim"]
    if case["kind"] == "rotate":
        t, hq = case["tokens"], case["heads_q"]
        # q, k read and written in bf16; dQ too, dK read in fp32; the table's rows that occur, the positions
        return {"bytes": t * d * (8 * hq + 4 * hkv + 6 * hkv) + 4 * t * (case["rot"] + case["axes"]),
                "flops": 6 * t * (hq + hkv) * case["rot"]}
    held, new = _lens(case)
    t = int(new.sum())
    if case["kind"] == "pages":
        branch, page, copied, entries = case["branch"], case["page"], 0, 0
        for a in range(0, case["seqs"], branch):
            writers = int((new[a:a + branch] > 0).sum())
            entries += branch * -(-int(held[a]) // page)
            if held[a] % page:        # the last of them keeps the page where nobody else holds it
                copied += writers - (writers == branch)
        return {"bytes": 8 * entries + copied * case["layers"] * 4 * hkv * (page * d + 4) + 24 * case["seqs"], "flops": 0}
    if case["kind"] == "compact":
        n = sum(len(k) for k in _kept(case, held, new))
        return {"bytes": 4 * n * hkv * d + 4 * n, "flops": 8 * n * hkv * d}
    hq = case["heads_q"]
    if case["kind"] != "tree":
        return {"bytes": t * (4 * hq * d + 4 * hkv * d + 2 * hkv * d + (2 * hkv * d if case["k_out"] else 0)
                              + 4 * case["rot"]),
                "flops": 3 * t * (hq + hkv) * case["rot"] + 4 * t * hkv * d}
    bits, depth = _tree_of(new, _parents(case, new), -(-int(new.max()) // 64))
    named = np.unpackbits(bits.view(np.uint8), axis=1).sum(1)
    at = np.concatenate([[0], np.cumsum(new)])
    w, sinks, pairs, tokens = case["window"], case["sinks"], 0, 0
    for i, (a, n) in enumerate(zip(held, new)):
        if not n:
            continue
        pos = int(a) + depth[at[i]:at[i + 1]]
        lo = np.minimum(int(a), np.maximum(0, pos - w + 1))
        pairs += int((int(a) - lo + np.minimum(lo, sinks)).sum() + np.minimum(named[at[i]:at[i + 1]], w + sinks).sum())
        tokens += int(a) - int(lo.min()) + min(int(lo.min()), sinks) + int(n)
    return {"bytes": 2 * tokens * hkv * d + 4 * t * hq * d + 4 * t * hq, "flops": 4 * d * hq * pairs}


# ---------------------------------------------------------------------------
# the operators from their definitions, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _exact_tree, "draft": _exact_new, "image": _exact_new, "rotate": _exact_rotate,
            "compact": _exact_compact, "pages": _exact_pages}[case["kind"]](s)


def _exact_tree(s):
    case = s["case"]
    held, new = _lens(case)
    hq, hkv, d, page = case["heads_q"], case["heads_kv"], case["dim"], case["page"]
    parents = _parents(case, new)
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((hq, s["total_new"]), dtype=torch.float64, device="cuda")
    at = 0
    for i in range(case["seqs"]):
        a, t = int(held[i]), int(new[i])
        if not t:
            continue
        pages = s["table"][i, :-(-(a + t) // page)].long()

        def tokens(name):
            val = s[name + "_codes"][pages].view(torch.float8_e4m3fn).to(torch.float32).double()
            val = val * s[name + "_scale"][pages].double()[..., None, None]
            return val.transpose(0, 1).reshape(hkv, -1, d)[:, :a + t]

        k, v = tokens("k"), tokens("v")
        see, place = np.zeros((t, a + t), dtype=bool), np.arange(a + t)
        for j in range(t):
            up, path = j, []
            while up >= 0:
                path.append(up)
                up = int(parents[at + up])
            place[a + j] = a + len(path) - 1
            see[j, :a] = True
            see[j, [a + x for x in path]] = True
        see &= (place[a:, None] - place[None] < case["window"]) | (place[None] < case["sinks"])
        see = torch.from_numpy(see).cuda()
        q = s["q"][at:at + t].double().view(t, hkv, hq // hkv, d).permute(1, 2, 0, 3)
        for g in range(hkv):
            sc = torch.where(see, s["scale"] * torch.matmul(q[g], k[g].t()), -math.inf)
            ls = torch.logsumexp(sc, -1)
            h = slice(g * (hq // hkv), (g + 1) * (hq // hkv))
            o[at:at + t, h] = torch.matmul(torch.exp(sc - ls[..., None]), v[g]).transpose(0, 1)
            lse[h, at:at + t] = ls
        at += t
    return [o, lse]


def _exact_turn(s, x, place, sign=1.0):
    """x [tokens, H, d] turned pair by pair; place [axes, tokens]."""
    case = s["case"]
    rot = case["rot"]
    y = x.double().clone()
    for p, axis in enumerate(s["axis"]):
        row = s["cos_sin"].double()[place[int(axis)].long()]
        c, z = row[:, p, None], sign * row[:, rot // 2 + p, None]
        a, b = (2 * p, 2 * p + 1) if case["interleaved"] else (p, p + rot // 2)
        u, w = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = u * c - w * z, w * c + u * z
    return y


def _round_e4m3(x):
    """Nearest e4m3 value (ties to even) of a 64-bit tensor, saturating."""
    x = x.clamp(-E4M3_MAX, E4M3_MAX)
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_write(s, values, name, where, slot):
    codes = s[name + "_codes"].view(torch.float8_e4m3fn).to(torch.float32).double()
    scales = s[name + "_scale"].double()
    at, slots = _cuda(where, np.int64), _cuda(slot, np.int64)
    top = torch.zeros_like(scales).index_reduce_(0, at, values.abs().amax(-1), "amax")
    need = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / E4M3_MAX)).clamp(MIN_EXP, MAX_EXP))
    pages, which = np.unique(where, return_index=True)   # (a page's tokens come in order)
    had, pg = _cuda(np.asarray(slot)[which], np.int64)[:, None], _cuda(pages, np.int64)
    grown = torch.where(had > 0, torch.maximum(need[pg], scales[pg]), need[pg])
    again = _round_e4m3(codes[pg] * (scales[pg] / grown)[..., None, None])
    keep = torch.arange(codes.shape[2], device="cuda")[None, None, :, None] < had[..., None, None]
    codes[pg] = torch.where(keep, again, codes[pg])
    scales[pg] = grown
    codes[at, :, slots] = _round_e4m3(values / scales[at][..., None])
    return [codes, scales]


def _exact_new(s):
    case = s["case"]
    held, new = _lens(case)
    seq = np.repeat(np.arange(case["seqs"]), new)
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(held, new)])
    place = s["positions"]
    if case["kind"] == "draft":
        place = _cuda(np.repeat(held, new) + _tree_of(new, s["parents"].cpu().numpy(), s["words"])[1])[None]
    k = _exact_turn(s, s["k"], place)
    where = s["table"].cpu().numpy()[seq, pos // case["page"]]
    out = [_exact_turn(s, s["q"], place)] + _exact_write(s, k, "k", where, pos % case["page"])
    out += _exact_write(s, s["v"].double(), "v", where, pos % case["page"])
    out += [k] if s["k_out"] is not None else []
    return out + ([None, None] if case["kind"] == "draft" else [])


def _exact_rotate(s):
    p = s["positions"]
    return [_exact_turn(s, s["q"], p), _exact_turn(s, s["k"], p), _exact_turn(s, s["d_q"], p, -1.0),
            _exact_turn(s, s["d_k"], p, -1.0)]


def _exact_compact(s):
    case = s["case"]
    held, new = _lens(case)
    kept = _kept(case, held, new)
    page, table = case["page"], s["table"].cpu().numpy()
    target = s["dst_table"].cpu().numpy() if "dst_table" in s else table
    seq = np.repeat(np.arange(case["seqs"]), [len(k) for k in kept])
    source = np.concatenate(kept)
    place = np.concatenate([a + np.arange(len(k)) for a, k in zip(held, kept)])
    of, slot = _cuda(table[seq, source // page], np.int64), _cuda(source % page, np.int64)
    out = []
    for x in "kv":
        codes = s[x + "_codes"].view(torch.float8_e4m3fn)[of, :, slot].to(torch.float32).double()
        out += _exact_write(s, codes * s[x + "_scale"].double()[of][..., None], x, target[seq, place // page], place % page)
    return out + [None]


def _exact_pages(s):
    """Row by row: what every sequence takes over, then, in order, a page of its own for each place that it writes."""
    case = s["case"]
    page = case["page"]
    table, refs = s["table"].tolist(), s["refs"].tolist()
    source, new, lens = s["source"].tolist(), s["new"].tolist(), s["committed"].tolist()
    after = [[p if c * page < lens[source[i]] else -1 for c, p in enumerate(table[source[i]])] for i in range(len(table))]
    for rows, by in ((after, 1), (table, -1)):
        for row in rows:
            for p in row:
                if p >= 0:
                    refs[p] += by
    free = [p for p, n in enumerate(refs) if n == 0]
    copies = []
    for i, row in enumerate(after):
        a = lens[source[i]]
        for c in range(a // page, -(-(a + new[i]) // page) if new[i] else 0):
            if row[c] >= 0 and refs[row[c]] == 1:
                continue
            p = free.pop(0)
            if row[c] >= 0:
                refs[row[c]] -= 1
                if c * page < a:
                    copies.append((row[c], p))
            row[c], refs[p] = p, 1
    out = [None] * 6
    for y in s["layers"]:
        for name in ("k_codes", "k_scale", "v_codes", "v_scale"):
            t = y[name].clone()
            for of, to in copies:
                t[to] = y[name][of]
            out.append(t.view(torch.float8_e4m3fn).to(torch.float64) if name.endswith("codes") else t.double())
    return out
