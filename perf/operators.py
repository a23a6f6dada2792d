"""Performance cases of the paged K/V cache: writing rows into its pages (quantised where the cache holds 8 bits), reading
them back, and the attention of new rows over it.

Position p of sequence b lives in page page_table[b][p // page_size] at slot p % page_size; an entry outside [0, n_pages) means
that there is no page. Pages are [n_pages, kv_heads, page_size, head_dim] in bf16, fp32 or e4m3; an e4m3 cache has one scale for
each position and K/V head, a power of two held as its exponent in 8 bits: the smallest of at least 2^-110 with which the row's
largest finite magnitude is at most 448.

  store  rows of new K and V go to their positions' slots
  load   the inverse: the rows at given positions, zeros for positions without a page
  attn   softmax(q K^T / sqrt(head_dim)) V over the positions below the sequence's length that have a page, zeros where the
         exponentials sum to zero

Where `own` is true the library's entry points are called, otherwise the same is computed with elementary torch operations.

    python -c "from perf import operators; print(operators.listed())"
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp32": 4, "e4m3": 1}
_LOWEST, _HIGHEST = -110, 120            # exponents of the scales


def _case(name, kind, batch, q_heads, kv_heads, seq_len, rows, cache, page, dtype="bf16", head_dim=128, ragged=False, holes=0.0):
    return {"name": name, "kind": kind, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "seq_len": seq_len, "rows": rows, "cache": cache, "page": page, "dtype": dtype, "ragged": ragged, "holes": holes}


def listed():
    return [
        # one new token of one sequence: the smallest call of a decode loop, nothing but latency
        _case("attn_one_token", "attn", 1, 32, 32, 512, 1, "bf16", 16),
        # a batch of decoding sequences at different lengths, grouped-query heads
        _case("attn_one_token_ragged", "attn", 16, 28, 4, 4096, 1, "bf16", 64, ragged=True),
        # two long documents: few (sequence, head) pairs, so the length has to be split
        _case("attn_one_token_long", "attn", 2, 28, 4, 131072, 1, "e4m3", 128),
        # a full batch of decoding sequences, the largest stream of keys and values
        _case("attn_one_token_batch", "attn", 32, 32, 32, 4096, 1, "e4m3", 64, ragged=True),
        # a denoising step: 32 active rows a sequence
        _case("attn_active_rows", "attn", 8, 32, 32, 1024, 32, "bf16", 16),
        # active sets of different sizes, grouped-query heads, sizes that divide nothing, some pages given back
        _case("attn_active_rows_ragged", "attn", 16, 28, 4, 769, 129, "e4m3", 32, ragged=True, holes=0.1),
        # a refresh of long sequences: every row attends to every position, bound by arithmetic
        _case("attn_refresh", "attn", 4, 32, 32, 1536, 1536, "e4m3", 64),
        # a toy model in fp32
        _case("attn_fp32", "attn", 3, 4, 4, 203, 17, "fp32", 16, dtype="fp32", head_dim=32),
        # what one denoising step writes
        _case("store_step", "store", 8, 32, 32, 1024, 8, "e4m3", 16),
        # prompts written at once
        _case("store_prompt", "store", 4, 32, 32, 1536, 1536, "e4m3", 64),
        # the same read back, to hand a sequence on
        _case("load_prompt", "load", 4, 32, 32, 1536, 1536, "e4m3", 64),
        # a few rows of an unquantised cache, some positions without a page
        _case("load_rows_ragged", "load", 16, 28, 4, 769, 77, "bf16", 32, ragged=True, holes=0.1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


def draw(rng):
    """One more case of the ranges above (no name)."""
    while True:
        kind = rng.choice(("attn", "attn", "attn", "store", "load"))
        dtype, head_dim = "bf16", rng.choice((128, 128, 128, 64))
        q_heads, kv_heads = rng.choice(((32, 32), (32, 32), (28, 4), (24, 8), (16, 1)))
        cache = rng.choice(("bf16", "e4m3", "e4m3"))
        if rng.random() < 0.15:
            dtype, head_dim, q_heads, kv_heads = "fp32", rng.choice((32, 64, 128)), 8, rng.choice((2, 8))
            cache = rng.choice(("fp32", "e4m3", "bf16") if kind != "attn" else ("fp32", "e4m3"))
        seq_len = _log_int(rng, 1, 131072)
        rows = 1 if kind == "attn" and rng.random() < 0.4 else _log_int(rng, 1, min(seq_len, 1536))
        c = _case("", kind, _log_int(rng, 1, 32), q_heads, kv_heads, seq_len, rows, cache, rng.choice((16, 32, 64, 128, 256)),
                  dtype, head_dim, rng.random() < 0.5, rng.choice((0.0, 0.0, 0.1)))
        cells = c["batch"] * kv_heads * seq_len * head_dim
        scores = c["batch"] * q_heads * rows * seq_len
        if cells > 32 * 32 * 4096 * 128 or scores > 3.1e8 or (dtype == "fp32" and scores * head_dim > 5e9) or work(c)["bytes"] > 5.6e8:
            continue
        del c["name"]
        return c


def _lengths(case):
    """Keys and rows of each sequence; ragged: from all of them down to a few."""
    B, L, R = case["batch"], case["seq_len"], case["rows"]
    share = [(B - b) / B if case["ragged"] else 1.0 for b in range(B)]
    keys = [max(1, math.ceil(L * s)) for s in share]
    return keys, [min(k, max(1, math.ceil(R * s))) for k, s in zip(keys, share)]


def _exponent(amax):
    """Exponent of the scale of rows with these largest magnitudes."""
    m, x = torch.frexp(amax)                                  # amax = m 2^x, m in [1/2, 1)
    e = x.to(torch.int32) - 9 + (m > 0.875).to(torch.int32)
    return torch.where(amax > 0, e, _LOWEST).clamp(_LOWEST, _HIGHEST)


def _quantise(x):
    """fp32 rows -> (e4m3 codes, exponents of their scales)."""
    fine = torch.isfinite(x)
    e = _exponent(torch.where(fine, x, 0.0).abs().amax(-1))
    most = torch.where(e == _HIGHEST, 240.0, 448.0)[..., None]
    y = x * ((127 - e) << 23).view(torch.float32)[..., None]
    y = torch.where(fine, torch.minimum(torch.maximum(y, -most), most), float("nan"))
    return y.to(torch.float8_e4m3fn), e


def _scale_values(scale):
    return (scale.view(torch.uint8).to(torch.int32) << 23).view(torch.float32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, Hq, Hkv, dh, L, S = (case[k] for k in ("batch", "q_heads", "kv_heads", "head_dim", "seq_len", "page"))
    keys, counts = _lengths(case)
    order = torch.randperm(B, generator=torch.Generator().manual_seed(seed)).tolist()
    keys, counts = [keys[i] for i in order], [counts[i] for i in order]
    act = _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    # each sequence has the pages for its positions, in any order; the table is as wide as the longest and a page more
    need = [-(-k // S) for k in keys]
    n_pages = sum(need) + max(2, sum(need) // 16)
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    width = max(need) + 1
    place = torch.arange(width, device="cuda")[None, :]
    needed = torch.tensor(need, device="cuda")[:, None]
    first = torch.tensor([sum(need[:b]) for b in range(B)], device="cuda")[:, None]
    table = torch.where(place < needed, ids[torch.where(place < needed, first + place, 0)], -1)
    given_back = torch.rand((B, width), generator=g, device="cuda") < case["holes"]
    table = torch.where(given_back & (place > 0), -1, table).to(torch.int32).contiguous()

    def pages():
        x = normal(n_pages, Hkv, S, dh) * (0.5 + torch.rand((Hkv, 1, dh), generator=g, device="cuda"))
        if case["cache"] != "e4m3":
            return x.to(_TYPES[case["cache"]]), None
        codes, e = _quantise(x)
        return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)

    s = {"page_table": table, "seq_len": torch.tensor(keys, dtype=torch.int32, device="cuda"), "kind": case["kind"]}
    s["k_pages"], s["k_scale"] = pages()
    s["v_pages"], s["v_scale"] = pages()
    # slots behind a sequence's end hold whatever was there before, here NaN
    tail = torch.tensor([k % S for k in keys], device="cuda")
    last = torch.gather(table, 1, needed - 1)[:, 0]
    for b in [b for b in range(B) if keys[b] % S and int(last[b]) >= 0]:
        for x in (s["k_pages"], s["v_pages"]):
            x.view(torch.uint8)[last[b], :, int(tail[b]):] = 0xFF
    R, most = sum(counts), max(counts)
    off = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    off[1:] = torch.tensor(counts, device="cuda").cumsum(0)
    s |= {"row_off": off, "rows": R, "max_rows": most}
    if case["kind"] == "attn":
        s["q"] = normal(R, Hq, dh).to(act)
        s["out"] = torch.zeros_like(s["q"])
        s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        return s
    # distinct positions of each sequence, ascending
    pick = torch.rand((B, L), generator=g, device="cuda")
    pick = torch.where(torch.arange(L, device="cuda")[None, :] < s["seq_len"][:, None], pick, 2.0).argsort(dim=1)
    taken = torch.zeros((B, L), dtype=torch.bool, device="cuda")
    taken.scatter_(1, pick, torch.arange(L, device="cuda")[None, :] < torch.tensor(counts, device="cuda")[:, None])
    s["pos"] = taken.nonzero()[:, 1].to(torch.int32).contiguous()
    if case["kind"] == "store":
        s["k"], s["v"] = normal(R, Hkv, dh).to(act), (2.0 * normal(R, Hkv, dh)).to(act)
    else:
        s["k"], s["v"] = (torch.zeros((R, Hkv, dh), dtype=act, device="cuda") for _ in range(2))
    return s


def _sequence_of_rows(s):
    return torch.searchsorted(s["row_off"][1:].contiguous(), torch.arange(s["rows"], device="cuda", dtype=torch.int32), right=True)


def _places(s):
    """Page and slot of each row's position, and whether it has a page."""
    S = s["k_pages"].shape[2]
    pos = s["pos"].long()
    page = s["page_table"][_sequence_of_rows(s), pos // S].long()
    there = (page >= 0) & (page < s["k_pages"].shape[0])
    return torch.where(there, page, 0), pos % S, there


def _store_rows(new, pages, scale, page, slot):
    if scale is None:
        pages[page, :, slot] = new.to(pages.dtype)
    else:
        codes, e = _quantise(new.float())
        pages.view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
        scale.view(torch.uint8)[page, :, slot] = (e + 127).to(torch.uint8)


def _store(s):
    page, slot, there = _places(s)
    _store_rows(s["k"][there], s["k_pages"], s["k_scale"], page[there], slot[there])
    _store_rows(s["v"][there], s["v_pages"], s["v_scale"], page[there], slot[there])


def _load_rows(out, pages, scale, page, slot, there):
    if scale is None:
        x = pages[page, :, slot].float()
    else:
        x = pages.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
        x = x * _scale_values(scale.view(torch.uint8)[page, :, slot])[..., None]
    out.copy_(torch.where(there[:, None, None], x, 0.0).to(out.dtype))


def _load(s):
    at = _places(s)
    _load_rows(s["k"], s["k_pages"], s["k_scale"], *at)
    _load_rows(s["v"], s["v_pages"], s["v_scale"], *at)


def _attend(s):
    q, table, off = s["q"], s["page_table"], s["row_off"].long()
    n_pages, Hkv, S, dh = s["k_pages"].shape
    R, Hq = q.shape[:2]
    B, width = table.shape
    there = (table >= 0) & (table < n_pages)
    at = torch.where(there, table, 0).long()
    seen = there.repeat_interleave(S, dim=1, output_size=width * S) & (torch.arange(width * S, device="cuda")[None, :] < s["seq_len"][:, None])

    def gathered(pages, scale):                      # [B, Hkv, keys, dh] in fp32, zeros where nothing is seen
        if scale is None:
            x = pages[at].float()
        else:
            x = pages.view(torch.uint8)[at].view(torch.float8_e4m3fn).float()
            x = x * _scale_values(scale.view(torch.uint8)[at])[..., None]
        x = x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, width * S, dh)
        return torch.where(seen[:, None, :, None], x, 0.0)

    seq, most = _sequence_of_rows(s), s["max_rows"]
    row = (off[:-1, None] + torch.arange(most, device="cuda")[None, :]).clamp(max=R - 1)      # rows of each sequence, padded
    x = q[row].float().view(B, most, Hkv, Hq // Hkv, dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * (Hq // Hkv), dh)
    scores = torch.matmul(x, gathered(s["k_pages"], s["k_scale"]).transpose(2, 3).contiguous()) / math.sqrt(dh)
    scores = torch.where(seen[:, None, None, :], scores, float("-inf"))
    e = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    total = e.sum(-1, keepdim=True)
    y = torch.matmul(e, gathered(s["v_pages"], s["v_scale"]))
    y = torch.where(total == 0, 0.0, y / total).view(B, Hkv, most, Hq // Hkv, dh).permute(0, 2, 1, 3, 4).reshape(B, most, Hq, dh)
    s["out"].copy_(y[seq, torch.arange(R, device="cuda") - off[seq]].to(q.dtype))


def run(state):
    s = state
    if own:
        import paper_2505_15781_amd as P
        cache = P.PagedCache(s["k_pages"], s["v_pages"], s["page_table"], s["seq_len"], s["k_scale"], s["v_scale"])
        if s["kind"] == "attn":
            P.paged_attn(cache, s["q"], s["row_off"], s["out"], s["max_rows"], s["workspace"])
        elif s["kind"] == "store":
            P.paged_store(cache, s["k"], s["v"], s["pos"], s["row_off"])
        else:
            P.paged_load(cache, s["k"], s["v"], s["pos"], s["row_off"])
    else:
        {"attn": _attend, "store": _store, "load": _load}[s["kind"]](s)
    if s["kind"] == "attn":
        return {"out": s["out"]}
    if s["kind"] == "load":
        return {"k": s["k"], "v": s["v"]}
    return {k: s[k] for k in ("k_pages", "v_pages", "k_scale", "v_scale") if s[k] is not None}


def work(case):
    keys, counts = _lengths(case)
    Hq, Hkv, dh = case["q_heads"], case["kv_heads"], case["head_dim"]
    held = 2.0 * Hkv * (dh * _BYTES[case["cache"]] + (1 if case["cache"] == "e4m3" else 0))      # K and V of a position
    es = _BYTES[case["dtype"]]
    if case["kind"] == "attn":
        return {"bytes": held * sum(keys) * (1.0 - case["holes"]) + 2.0 * sum(counts) * Hq * dh * es,
                "flops": sum(4.0 * Hq * dh * k * r for k, r in zip(keys, counts)) * (1.0 - case["holes"])}
    rows = sum(counts) * (1.0 - case["holes"])
    return {"bytes": rows * (held + 2.0 * Hkv * dh * es + 4), "flops": 2.0 * rows * Hkv * dh}


def exact(case, seed):
    """The same from the definitions, position by position's page, in 64 bits."""
    s = prepare(case, seed)
    n_pages, Hkv, S, dh = s["k_pages"].shape
    table, off, keys = s["page_table"].tolist(), s["row_off"].tolist(), s["seq_len"].tolist()

    def values(pages, scale, ids):                   # [Hkv, len(ids) * S, dh]
        ids = torch.tensor(ids, device="cuda")
        if scale is None:
            x = pages[ids].double()
        else:
            power = scale.view(torch.uint8)[ids].double() - 127.0
            x = pages.view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * torch.exp2(power)[..., None]
        return x.transpose(0, 1).reshape(Hkv, -1, dh)

    if case["kind"] == "attn":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        group = case["q_heads"] // Hkv
        for b, n in enumerate(keys):
            held = [(j, p) for j, p in enumerate(table[b]) if 0 <= p < n_pages and j * S < n]
            if not held:
                continue
            at = (torch.tensor([j for j, _ in held], device="cuda")[:, None] * S + torch.arange(S, device="cuda")).reshape(-1)
            k, v = (values(s[x + "_pages"], s[x + "_scale"], [p for _, p in held])[:, at < n] for x in "kv")
            for h in range(case["q_heads"]):
                z = s["q"][off[b]:off[b + 1], h].double() @ k[h // group].T.contiguous() / math.sqrt(dh)
                out[off[b]:off[b + 1], h] = torch.softmax(z, dim=-1) @ v[h // group]
        return {"out": out}
    pos = s["pos"].long()
    seq = torch.repeat_interleave(torch.arange(len(keys), device="cuda"), torch.diff(s["row_off"]).long())
    page = s["page_table"].long()[seq, torch.div(pos, S, rounding_mode="floor")]
    ok = (page >= 0) & (page < n_pages)
    page, slot = page[ok], (pos % S)[ok]
    got = {}
    for x in "kv":
        pages, scale, rows = s[x + "_pages"], s[x + "_scale"], s[x]
        if case["kind"] == "load":
            y = torch.zeros(rows.shape, dtype=torch.float64, device="cuda")
            y[ok] = pages.double()[page, :, slot]
            if scale is not None:
                y[ok] *= torch.exp2(scale.view(torch.uint8).double() - 127.0)[page, :, slot][..., None]
            got[x] = y
            continue
        y, held = rows[ok].double(), pages.double()
        if scale is None:
            held[page, :, slot] = y
        else:
            e = torch.ceil(torch.log2(y.abs().amax(-1).clamp(min=1e-300) / 448.0)).clamp(-110, 120)
            z = y / torch.exp2(e)[..., None]
            step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)         # distance of neighbouring e4m3 values
            held[page, :, slot] = torch.round(z / step) * step
            powers = torch.exp2(scale.view(torch.uint8).double() - 127.0)
            powers[page, :, slot] = torch.exp2(e)
            got[x + "_scale"] = powers
        got[x + "_pages"] = held
    return got
