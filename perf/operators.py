"""The operators that keep a reduced cache in few bits and answer new tokens from it, and what they are measured on.

* ``write``   kept rows of a K/V cache are quantised as the reduced cache is written, and read back; or the rows of newly
              generated tokens are appended to it (``kvcrush_quantize``, ``kvcrush_dequantize``);
* ``attend``  attention of new tokens over a cache, 16-bit, float32 or quantised: one token for each sequence, or a tree of
              drafted tokens with keys and values of their own (``kvcrush_attend``);
* ``pages``   a new token attends to the pages whose bounds promise the largest logits (``kvcrush_page_bounds``,
              ``kvcrush_attend_pages``).

Sizes are those of the package's workloads (``inputs.paper_workloads``: heads, prompts, the ragged batch), of its paged setting
(pages of 32 and chunks of 8 tokens) and of reduced caches at a quarter of a prompt; ``draw`` spreads over the ranges
between them.  With ``own`` false everything is computed by elementary operations in float32 or float64.
"""
import math

import numpy as np
import torch

from paper_2503_00022_b200 import inputs

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ITEM = {"bf16": 2.0, "fp16": 2.0, "fp32": 4.0, "int8": 1.0, "e4m3": 1.0, "int4": 0.5}
PARAMS = {"int8": 4, "e4m3": 4, "int4": 8}                         # bytes of a row's scale, or scale and zero
TOP = {"int8": 127.0, "e4m3": 448.0, "int4": 15.0}                 # codes a row's scale spans
TINY = 2.0 ** -126                                                 # smaller scales count as zero


def _case(name, kind, layers, q_heads, kv_heads, dim, lens, dtype, fmt="", kept=0.0, new=0, page=0, budget=0, fresh=False):
    """lens: tokens of each sequence in the cache; fmt: type of the cache when it is not dtype; kept: share of the rows that
    is written; new: drafted tokens of a sequence (0: one token that is in the cache already); page, budget: page size and
    pages that a query reads; fresh: the pages' bounds are computed for the whole prompt, otherwise for the last page."""
    return {"name": name, "kind": kind, "layers": layers, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "lens": ",".join(str(int(x)) for x in lens), "dtype": dtype, "fmt": fmt, "kept": kept, "new": new, "page": page,
            "budget": budget, "fresh": fresh}


def listed():
    ragged = inputs.paper_workloads()["cfg5_ragged_batch16"].seqlens
    return [
        # the tokens just generated by a batch of 16 are appended to an 8-bit float cache: the smallest write
        _case("append_e4m3", "write", 32, 32, 8, 128, [1] * 16, "bf16", fmt="e4m3"),
        # a quarter of a long prompt is kept, in 8 bits, over the whole stack of layers: the largest write
        _case("write_8k_int8", "write", 32, 32, 32, 128, [8192], "bf16", fmt="int8", kept=0.25),
        # 16 ragged prompts, half of them kept in 4 bits, float16 and heads of 96
        _case("write_ragged_int4", "write", 8, 32, 8, 96, ragged, "fp16", fmt="int4", kept=0.5),
        # one generated token over a reduced cache of 2048 rows, one layer: the smallest attention call
        _case("token_2k", "attend", 1, 32, 8, 128, [2048], "bf16"),
        # one token for each of 16 ragged sequences over 8-bit caches
        _case("token_batch_int8", "attend", 1, 32, 8, 128, ragged, "bf16", fmt="int8"),
        # one token over the longest cache, held in 4 bits
        _case("token_32k_int4", "attend", 1, 32, 8, 128, [32768], "bf16", fmt="int4"),
        # a drafted tree of 15 tokens for each of 16 ragged sequences, one query head a KV head, heads of 96
        _case("tree_batch_fp16", "attend", 1, 32, 32, 96, ragged, "fp16", new=15),
        # a tree of 63 tokens over the longest cache, grouped-query heads: the largest attention call
        _case("tree_32k", "attend", 1, 32, 8, 128, [32768], "bf16", new=63),
        # a small model in float32: a short chain of drafts over an odd length
        _case("tree_fp32", "attend", 1, 8, 8, 64, [1001], "fp32", new=7),
        # a generated token reads 64 pages of 32 of the longest cache
        _case("pages_32k", "pages", 1, 32, 8, 128, [32768], "bf16", page=32, budget=64),
        # the ragged batch in chunks of 8, an 8-bit cache
        _case("pages_batch_int8", "pages", 1, 32, 8, 128, ragged, "fp16", fmt="int8", page=8, budget=96),
        # the first token after a prompt: bounds of the whole prompt, then its pages
        _case("pages_fresh_8k", "pages", 1, 32, 32, 128, [8191], "bf16", page=32, budget=32, fresh=True),
    ]


MOST_BYTES, MOST_FLOPS = 3.2e9, 3.3e10                             # no drawn case costs more than the largest listed one


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["write", "attend", "attend", "pages"])
        q_heads, kv_heads = rng.choice([(8, 8), (32, 32), (32, 8), (32, 8), (32, 4), (40, 40), (24, 2)])
        dim = rng.choice([64, 96, 128, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp16"])
        fmt = rng.choice(["int8", "e4m3", "int4"])
        n_seqs = rng.choice([1, 1, _log_int(rng, 2, 16)])
        longest = _log_int(rng, 200, 32768)
        layers, kept, new, page, budget, fresh = rng.choice([1, 1, 2]), 0.0, 0, 0, 0, False
        if kind == "write":
            layers, kept = _log_int(rng, 1, 32), round(rng.uniform(0.1, 0.9), 3)
            if rng.random() < 0.25:
                longest, kept = _log_int(rng, 1, 16), 0.0
        elif kind == "attend":
            fmt = rng.choice(["", fmt])
            longest = _log_int(rng, 30, 32768)
            new = rng.choice([0, 0, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
            if rng.random() < 0.1:
                q_heads, kv_heads, dtype, fmt, longest, new = 8, 8, "fp32", "", min(longest, 4096), min(new, 16)
        else:
            fmt = rng.choice(["", "", fmt])
            page, fresh = rng.choice([8, 16, 32, 64]), rng.random() < 0.3
            budget = max(2, int(rng.uniform(0.05, 0.5) * longest / page))
        lens = [longest] + [max(1, int(longest * rng.uniform(0.25, 1.0))) for _ in range(n_seqs - 1)]
        c = _case("", kind, layers, q_heads, kv_heads, dim, lens, dtype, fmt, kept, new, page, budget, fresh)
        del c["name"]
        w = work(c)
        held = layers * sum(lens) * kv_heads * dim * 4 * 2         # both tensors in float32, as the plain form holds them
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS and held <= 8e9:
            return c


def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _kept(case):
    return [max(1, int(case["kept"] * n)) if case["kept"] else n for n in _lens(case)]


def _pages(case):
    return [-(-n // case["page"]) for n in _lens(case)]


INITIAL, RECENT = 1, 2                                             # pages read by decree


# ---- inputs ------------------------------------------------------------------------------------------------------

def _rows(g, case, dev, is_key, lens=None):
    """Rows [layers, tokens, heads, dim] of a cache: normal values; keys carry attention sinks and heavy hitters."""
    lens = lens or _lens(case)
    out = torch.empty((case["layers"], sum(lens), case["kv_heads"], case["dim"]), dtype=DTYPES[case["dtype"]], device=dev)
    first = torch.cat([torch.arange(n, device=dev) for n in lens]) < inputs.SINK_TOKENS
    for x in out:
        v = torch.randn(x.shape, generator=g, device=dev)
        if is_key:
            heavy = torch.rand(len(first), generator=g, device=dev) < 0.05
            gain = torch.where(first, inputs.SINK_GAIN, torch.where(heavy, inputs.HEAVY_GAIN, 1.0))
            v *= gain[:, None, None]
        x.copy_(v)
    return out


def _tree(rng, n, words):
    """Mask words of a drafted tree: a token sees itself and its ancestors."""
    sees = np.zeros((n, n), dtype=bool)
    for i in range(n):
        if i:
            sees[i] = sees[rng.integers(max(0, i - 6), i)]
        sees[i, i] = True
    bits = np.zeros((n, words * 32), dtype=np.uint64)
    bits[:, :n] = sees
    return (bits.reshape(n, words, 32) << np.arange(32, dtype=np.uint64)).sum(axis=2).astype(np.uint32).view(np.int32)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    layers, hq, hk, dim, lens = case["layers"], case["q_heads"], case["kv_heads"], case["dim"], _lens(case)
    S, T, dt = len(lens), sum(lens), DTYPES[case["dtype"]]
    st = {"case": case}
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    st["starts"], st["lens"] = torch.from_numpy(cu[:-1]).to(dev), torch.tensor(lens, device=dev)
    if case["kind"] == "write":
        st["k"], st["v"] = _rows(g, case, dev, True), _rows(g, case, dev, False)
        kept = _kept(case)
        if case["kept"]:
            # kept tokens of every layer and sequence, ascending, and where they start in the list
            ids = [np.sort(rng.permutation(n)[:m]) for _ in range(layers) for n, m in zip(lens, kept)]
            st["idx"] = torch.from_numpy(np.concatenate(ids).astype(np.int32)).to(dev)
            rows, at, begin = sum(kept), np.tile(kept, layers), None
            st["cu_kept"] = torch.from_numpy(np.concatenate([[0], np.cumsum(at)]).astype(np.int32)).to(dev)
            owner = np.repeat(np.tile(cu[:-1], layers), at)
            st["source"] = (st["idx"].long() + torch.from_numpy(owner).to(dev)).view(layers, rows)
            st["place"] = torch.arange(rows, device=dev).expand(layers, rows).contiguous()
            st["rows"] = rows
        else:
            # appended behind what each sequence's part of the cache holds already
            room = 64 + max(lens)
            begin = np.stack([np.arange(S) * room + rng.integers(0, 64, S) for _ in range(layers)])
            st["rows"], st["begin"] = S * room, torch.from_numpy(begin.astype(np.int32)).to(dev)
            st["source"] = torch.arange(T, device=dev).expand(layers, T).contiguous()
            inside = np.concatenate([np.arange(n) for n in lens])
            st["place"] = torch.from_numpy(np.repeat(begin, lens, axis=1) + inside).to(dev)
        n = st["source"].shape[1]
        st["back"] = [torch.empty((layers, n, hk, dim), dtype=dt, device=dev) for _ in range(2)]
        st["cache"] = [_room(case, layers, st["rows"], dev) for _ in range(2)]
    else:
        k, v = _rows(g, case, dev, True), _rows(g, case, dev, False)
        counts = [case["new"] or 1] * S
        N = sum(counts)
        st["q"] = torch.randn((layers, N, hq, dim), generator=g, device=dev).to(dt)
        st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty((layers, hq, N), dtype=torch.float32, device=dev)
        st["k"], st["v"] = (_encode(x, case["fmt"]) for x in (k, v)) if case["fmt"] else (k, v)
        if case["new"]:
            words = -(-case["new"] // 32)
            st["mask"] = torch.from_numpy(np.concatenate([_tree(rng, n, words) for n in counts])).to(dev)
            st["k_new"], st["v_new"] = _rows(g, case, dev, False, counts), _rows(g, case, dev, False, counts)
        if case["kind"] == "pages":
            st["dense_k"] = k
            st["max_pages"] = max(_pages(case))
            st["lo"], st["hi"] = _bounds(st, k)
            shape = (layers, S, hk, min(case["budget"], st["max_pages"]))
            st["page_idx"] = torch.empty(shape, dtype=torch.int32, device=dev)
            st["n_pages"] = torch.empty(shape[:3], dtype=torch.int32, device=dev)
    if own:
        from paper_2503_00022_b200 import binding as kv
        st["prob"] = kv.Problem(layers, hq, hk, dim, lens, device=dev)
        st["status"] = torch.zeros(4, dtype=torch.int32, device=dev)
        if case["kind"] == "write":
            st["prob_kept"] = kv.Problem(layers, hq, hk, dim, _kept(case), device=dev)    # the reduced cache
            st["cache_q"] = [kv.QuantTensor(c, s, _code(kv, case["fmt"])) for c, s in st["cache"]]
        else:
            st["new"] = kv.NewTokens([case["new"] or 1] * S, mask=st.get("mask"), device=dev)
            if case["fmt"]:
                st["k"], st["v"] = (kv.QuantTensor(c, s, _code(kv, case["fmt"])) for c, s in (st["k"], st["v"]))
    return st


def _code(kv, fmt):
    return {"int8": kv.INT8, "e4m3": kv.E4M3, "int4": kv.INT4}[fmt]


def _room(case, layers, rows, dev):
    """Codes [layers, rows, heads, bytes] and scales [layers, rows, heads(, 2)] of a quantised cache; the scales of a head lie
    side by side."""
    width = case["dim"] // 2 if case["fmt"] == "int4" else case["dim"]
    codes = torch.zeros((layers, rows, case["kv_heads"], width), dtype=torch.uint8, device=dev)
    pair = (2,) if case["fmt"] == "int4" else ()
    return codes, torch.zeros((layers, case["kv_heads"], rows) + pair, dtype=torch.float32, device=dev).transpose(1, 2)


# ---- plain forms -------------------------------------------------------------------------------------------------

def _encode(x, fmt):
    """Codes and scales of rows x [..., dim].  The quotients are taken in float64: rows of few significant bits have many that
    lie on the border between two codes exactly."""
    x = x.float()
    zero = x.amin(-1) if fmt == "int4" else None
    span = x.amax(-1) - zero if fmt == "int4" else x.abs().amax(-1)
    scale = span * torch.tensor(1.0 / TOP[fmt], dtype=torch.float32, device=x.device)
    scale = torch.where(scale < TINY, torch.zeros_like(scale), scale)
    y = x.double() if zero is None else x.double() - zero[..., None].double()
    y = torch.where(scale[..., None] > 0, y * TOP[fmt] / span[..., None].double(), 0.0)
    if fmt == "int8":
        return y.round_().clamp_(-127, 127).to(torch.int8).view(torch.uint8), _by_head(scale)
    if fmt == "e4m3":
        # ties of the 8-bit float are exact in float32, which is rounded to first
        return y.clamp_(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8), _by_head(scale)
    n = y.round_().clamp_(0, 15).to(torch.uint8)
    return n[..., 0::2] | (n[..., 1::2] << 4), _by_head(torch.stack([scale, zero], dim=-1))


def _by_head(scale):
    """[layers, rows, heads(, 2)] with the scales of a head side by side."""
    return scale.transpose(1, 2).contiguous().transpose(1, 2)


def _values(cache, fmt):
    """The float32 values that codes stand for."""
    codes, scale = cache
    if fmt == "int8":
        return codes.view(torch.int8).float() * scale[..., None]
    if fmt == "e4m3":
        return codes.view(torch.float8_e4m3fn).float() * scale[..., None]
    n = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).float()
    return n * scale[..., 0:1] + scale[..., 1:2]


def _take(x, at):
    """Rows at[layer, i] of every layer of x [layers, rows, ...]."""
    return x[torch.arange(x.shape[0], device=x.device)[:, None], at]


def _padded(starts, lens, longest):
    """Row numbers [sequences, longest] and which of them exist."""
    at = torch.arange(longest, device=starts.device)
    there = at < lens[:, None]
    return torch.where(there, starts[:, None] + at, 0), there


def _write(st):
    case, layer = st["case"], torch.arange(st["source"].shape[0], device=st["source"].device)[:, None]
    out = []
    for x, (codes, scales) in ((st["k"], st["cache"][0]), (st["v"], st["cache"][1])):
        c, s = _encode(_take(x, st["source"]), case["fmt"])
        codes[layer, st["place"]], scales[layer, st["place"]] = c, s
        out += [_values((c, s), case["fmt"]).to(DTYPES[case["dtype"]]), s]
    return {"k": out[0], "v": out[2], "k_scale": out[1], "v_scale": out[3]}


def _attend(st, seen=None):
    """Attention of all new tokens; seen: which cached tokens a token of each sequence and KV head may see."""
    case = st["case"]
    layers, hk, dim, lens = case["layers"], case["kv_heads"], case["dim"], _lens(case)
    S, n = len(lens), case["new"] or 1
    G = case["q_heads"] // hk
    k, v = (_values(x, case["fmt"]) if case["fmt"] else x.float() for x in (st["k"], st["v"]))
    at, there = _padded(st["starts"], st["lens"], max(lens))
    k, v = k[:, at], v[:, at]                                      # [layers, S, longest, hk, dim]
    see = there[None, :, None, None, None, :] if seen is None else seen[:, :, :, None, None, :]
    if case["new"]:
        k = torch.cat([k, st["k_new"].float().view(layers, S, n, hk, dim)], dim=2)
        v = torch.cat([v, st["v_new"].float().view(layers, S, n, hk, dim)], dim=2)
        j = torch.arange(n, device=k.device)
        own_bits = ((st["mask"].view(S, n, -1)[:, :, j // 32] >> (j % 32)) & 1).bool()
        see = see.expand(-1, -1, -1, -1, n, -1)
        see = torch.cat([see, own_bits[None, :, None, None].expand(see.shape[0], -1, see.shape[2], -1, -1, -1)], dim=-1)
    q = st["q"].float().view(layers, S, n, hk, G, dim).permute(0, 1, 3, 4, 2, 5)
    x = torch.matmul(q.reshape(layers, S, hk, G * n, dim), k.permute(0, 1, 3, 4, 2)).view(layers, S, hk, G, n, -1)
    x = torch.where(see, x * (1.0 / math.sqrt(dim)), -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(layers, S, hk, G * n, -1), v.transpose(2, 3)).view(layers, S, hk, G, n, dim)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 1, 4, 2, 3, 5)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 3, 1, 4)
    st["out"].copy_(o.reshape(st["out"].shape))
    st["lse"].copy_(lse.reshape(st["lse"].shape))
    return {"out": st["out"], "lse": st["lse"]}


def _bounds(st, k):
    """Least and largest value of each channel in every page [layers, S * max_pages, hk, dim]; 0 where there is no page."""
    case, most = st["case"], st["max_pages"]
    at, there = _padded(st["starts"], st["lens"], most * case["page"])
    shape = (case["layers"], len(_lens(case)), most, case["page"], case["kv_heads"], case["dim"])
    x, there = k[:, at].view(shape), there.view(1, shape[1], most, case["page"], 1, 1)
    lo, hi = (torch.where(there, x, f).amin(3) if f > 0 else torch.where(there, x, f).amax(3) for f in (math.inf, -math.inf))
    some = there[:, :, :, 0]
    return tuple(torch.where(some, y, 0).to(k.dtype).flatten(1, 2) for y in (lo, hi))


def _refresh(st):
    """The bounds of the last page of every sequence, from its keys."""
    case, most = st["case"], st["max_pages"]
    last = (st["lens"] - 1) // case["page"]
    at, there = _padded(st["starts"] + last * case["page"], st["lens"] - last * case["page"], case["page"])
    x, there = st["dense_k"][:, at], there[None, :, :, None, None]
    rows = torch.arange(len(last), device=last.device) * most + last
    st["lo"][:, rows] = torch.where(there, x, math.inf).amin(2).to(x.dtype)
    st["hi"][:, rows] = torch.where(there, x, -math.inf).amax(2).to(x.dtype)


def _select(st):
    """Pages of the largest scores for every sequence and KV head, ascending, and which tokens they hold."""
    case, most = st["case"], st["max_pages"]
    layers, hk, S = case["layers"], case["kv_heads"], len(_lens(case))
    q = st["q"].double().view(layers, S, hk, -1, case["dim"])
    up, down = q.clamp(min=0).sum(3)[:, :, None], q.clamp(max=0).sum(3)[:, :, None]
    lo, hi = (st[b].double().view(layers, S, most, hk, case["dim"]) for b in ("lo", "hi"))
    score = (hi * up + lo * down).sum(-1).transpose(2, 3)           # [layers, S, hk, pages]
    page, count = torch.arange(most, device=score.device), -(-st["lens"] // case["page"])
    real = page < count[:, None]
    decreed = (page < INITIAL) | (page >= (count - RECENT)[:, None])
    score = torch.where(decreed[None, :, None], math.inf, score)
    score = torch.where(real[None, :, None], score, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :min(case["budget"], most)]
    taken = torch.arange(order.shape[-1], device=order.device) < count[:, None].clamp(max=order.shape[-1])
    taken = taken[None, :, None].expand(order.shape)
    chosen = torch.zeros(score.shape, dtype=torch.bool, device=score.device).scatter_(-1, order, taken)
    listed_pages = torch.sort(torch.where(taken, order, 1 << 30), dim=-1).values
    st["page_idx"].copy_(torch.where(taken, listed_pages, -1))
    st["n_pages"].copy_(taken.sum(-1))
    token = torch.arange(max(_lens(case)), device=score.device)
    return chosen[..., token // case["page"]] & (token < st["lens"][:, None])[None, :, None]


def run(st):
    case = st["case"]
    if own:
        return _run_own(st, case)
    if case["kind"] == "write":
        return _write(st)
    if case["kind"] == "attend":
        return _attend(st)
    if case["fresh"]:
        st["lo"], st["hi"] = _bounds(st, st["dense_k"])
    else:
        _refresh(st)
    return {**_attend(st, _select(st)), "pages": st["page_idx"], "n_pages": st["n_pages"], "lo": st["lo"], "hi": st["hi"]}


def _run_own(st, case):
    from paper_2503_00022_b200 import binding as kv
    prob, status = st["prob"], st["status"]
    if case["kind"] == "write":
        kq, vq = st["cache_q"]
        k, v = st["back"]
        if case["kept"]:
            total = case["layers"] * st["rows"]
            kv.kvcrush_quantize(prob, st["k"], st["v"], kq, vq, cu_kept=st["cu_kept"], idx=st["idx"], total_kept=total, status=status)
            kv.kvcrush_dequantize(st["prob_kept"], kq, vq, k, v, status=status)
            return {"k": k, "v": v, "k_scale": kq.scales, "v_scale": vq.scales}
        kv.kvcrush_quantize(prob, st["k"], st["v"], kq, vq, out_begin=st["begin"], status=status)
        kv.kvcrush_dequantize(prob, kq, vq, k, v, in_begin=st["begin"], status=status)
        return {"k": k, "v": v, "k_scale": _take(kq.scales, st["place"]), "v_scale": _take(vq.scales, st["place"])}
    if case["kind"] == "attend":
        kv.kvcrush_attend(prob, st["new"], st["q"], st["k"], st["v"], st["out"], k_new=st.get("k_new"), v_new=st.get("v_new"),
                          lse=st["lse"], status=status)
        return {"out": st["out"], "lse": st["lse"]}
    kv.kvcrush_page_bounds(prob, st["dense_k"], case["page"], st["lo"], st["hi"], recent_pages=0 if case["fresh"] else 1,
                           status=status)
    kv.kvcrush_attend_pages(prob, st["new"], st["q"], st["k"], st["v"], case["page"], st["lo"], st["hi"],
                            st["page_idx"].shape[-1], st["out"], keep_initial=INITIAL, keep_recent=RECENT,
                            page_idx=st["page_idx"], n_pages=st["n_pages"], lse=st["lse"], status=status)
    return {"out": st["out"], "lse": st["lse"], "pages": st["page_idx"], "n_pages": st["n_pages"], "lo": st["lo"], "hi": st["hi"]}


def work(case):
    layers, hq, hk, dim, lens, eb = (case[x] for x in ("layers", "q_heads", "kv_heads", "dim", "lens", "dtype"))
    lens, eb = _lens(case), ITEM[case["dtype"]]
    row = dim * ITEM[case["fmt"]] + PARAMS[case["fmt"]] if case["fmt"] else dim * eb
    T, S = sum(lens), len(lens)
    if case["kind"] == "write":
        # both tensors: rows read, codes and scales written, read again, values written
        n = 2.0 * layers * sum(_kept(case)) * hk
        return {"bytes": n * (2 * dim * eb + 2 * row) + (4 * n / hk / 2 if case["kept"] else 0), "flops": n * dim * 4}
    n = case["new"] or 1
    if case["kind"] == "attend":
        fresh = 2.0 * layers * S * n * (hq + (hk if case["new"] else 0)) * dim * eb + 4.0 * layers * hq * S * n
        return {"bytes": 2.0 * layers * T * hk * row + fresh,
                "flops": 4.0 * layers * hq * dim * n * (T + (S * n / 2 if case["new"] else 0))}
    pages = sum(_pages(case))
    read = sum(min(L, min(case["budget"], p) * case["page"]) for L, p in zip(lens, _pages(case)))
    bounds = 2.0 * layers * pages * hk * dim * eb
    made = layers * hk * dim * eb * (T if case["fresh"] else S * case["page"] / 2)
    listed_bytes = 4.0 * layers * S * hk * (min(case["budget"], max(_pages(case))) + 1)
    return {"bytes": bounds + made + 2.0 * layers * read * hk * row + 2.0 * layers * S * hq * dim * eb + listed_bytes,
            "flops": 4.0 * layers * hq * dim * read + 4.0 * layers * hk * dim * pages}


# ---- the definitions in 64 bits, one sequence and head at a time ---------------------------------------------------------

def _encode64(x, fmt):
    """(values, scales) of rows x in float64."""
    x = x.double()
    base = x.min(-1, keepdim=True).values if fmt == "int4" else torch.zeros_like(x[..., :1])
    scale = (x - base).abs().max(-1, keepdim=True).values / TOP[fmt]
    y = torch.where(scale > 0, (x - base) * TOP[fmt] / (x - base).abs().max(-1, keepdim=True).values, torch.zeros_like(x))
    if fmt == "e4m3":
        step = torch.exp2(torch.frexp(y).exponent.clamp(min=-5).double() - 4)    # three bits behind the leading one
        code = torch.round(y / step) * step
    else:
        code = torch.round(y)
    return base + scale * code, torch.cat([scale, base], -1) if fmt == "int4" else scale[..., 0]


def _cache64(cache, fmt):
    """Values of given codes in float64."""
    if not fmt:
        return cache.double()
    codes, scale = cache
    scale = scale.double()
    if fmt == "int4":
        n = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.float64, device=codes.device)
        n[..., 0::2], n[..., 1::2] = codes % 16, codes // 16
        return scale[..., 1:] + scale[..., :1] * n
    return codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).double() * scale[..., None]


def _softmax64(q, k, v):
    """(output, log-sum-exp) of one head: q [n, dim], k and v [n or 1, L, dim]."""
    x = torch.einsum("nd,nld->nl", q, k.expand(len(q), -1, -1)) / math.sqrt(q.shape[-1])
    lse = torch.logsumexp(x, -1)
    return torch.einsum("nl,nld->nd", torch.exp(x - lse[:, None]), v.expand(len(q), -1, -1)), lse


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    layers, hk, fmt, lens = case["layers"], case["kv_heads"], case["fmt"], _lens(case)
    if case["kind"] == "write":
        out = {}
        for name in "kv":
            got = [_encode64(st[name][i, st["source"][i]], fmt) for i in range(layers)]
            out[name], out[name + "_scale"] = torch.stack([a for a, _ in got]), torch.stack([b for _, b in got])
        return out
    G, n = case["q_heads"] // hk, case["new"] or 1
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
    if case["kind"] == "pages":
        pages = torch.full(st["page_idx"].shape, -1)
        n_pages = torch.zeros(st["n_pages"].shape, dtype=torch.int64)
        bounds = [torch.zeros(st["lo"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    begin = 0
    for s, L in enumerate(lens):
        rows = slice(begin, begin + L)
        begin += L
        pick = lambda c: (c[0][:, rows], c[1][:, rows]) if fmt else c[:, rows]   # noqa: E731
        k, v, new = _cache64(pick(st["k"]), fmt), _cache64(pick(st["v"]), fmt), slice(s * n, s * n + n)
        if case["new"]:
            bits = st["mask"][new].cpu().numpy().view(np.uint32)
            sees = torch.from_numpy(np.unpackbits(bits.view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)).cuda()
        for layer in range(layers):
            for h in range(hk):
                q = st["q"][layer, new, h * G:(h + 1) * G].double()
                kh, vh = k[layer, :, h], v[layer, :, h]
                if case["kind"] == "pages":
                    P, size = -(-L // case["page"]), case["page"]
                    full = torch.nn.functional.pad(st["dense_k"][layer, rows, h].double(), (0, 0, 0, P * size - L), value=math.nan)
                    full = full.view(P, size, -1)
                    low, high = full.nan_to_num(nan=math.inf).amin(1), full.nan_to_num(nan=-math.inf).amax(1)
                    at = slice(s * st["max_pages"], s * st["max_pages"] + P)
                    bounds[0][layer, at, h], bounds[1][layer, at, h] = low, high
                    score = torch.maximum(q[0, :, None] * low, q[0, :, None] * high).sum((0, 2))
                    score[:INITIAL] = math.inf
                    score[max(0, P - RECENT):] = math.inf
                    best = torch.argsort(score, descending=True, stable=True)[:pages.shape[-1]].sort().values
                    pages[layer, s, h, :len(best)], n_pages[layer, s, h] = best.cpu(), len(best)
                    tokens = (best[:, None] * size + torch.arange(size, device="cuda")).flatten()
                    tokens = tokens[tokens < L]
                    kh, vh = kh[tokens], vh[tokens]
                for i in range(G):
                    ki, vi = kh[None], vh[None]
                    if case["new"]:
                        x = torch.einsum("nd,ld->nl", q[:, i], torch.cat([kh, st["k_new"][layer, new, h].double()])) / math.sqrt(case["dim"])
                        x[:, L:][~sees] = -math.inf
                        total = torch.logsumexp(x, -1)
                        o = torch.exp(x - total[:, None]) @ torch.cat([vh, st["v_new"][layer, new, h].double()])
                    else:
                        o, total = _softmax64(q[:, i], ki, vi)
                    out[layer, new, h * G + i], lse[layer, h * G + i, new] = o, total
    if case["kind"] == "pages":
        return {"out": out, "lse": lse, "pages": pages, "n_pages": n_pages, "lo": bounds[0], "hi": bounds[1]}
    return {"out": out, "lse": lse}
