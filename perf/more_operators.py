"""Performance cases of what a server does around and over a paged K/V cache in 4 bits: pages for sequences that grow and leave, rotary
positions of new rows, their store and load, and the attention over the cache.

Position p of sequence b lives in page page_table[b][p // page_size] at slot p % page_size; an entry outside [0, n_pages) means that
there is no page. A cache in 4 bits holds two e2m1 codes to a byte, the lower dim in the lower four bits, and one scale for each 32 dims
of a row, a power of two held as its biased exponent in 8 bits: the smallest of at least 2^-110 with which the block's largest
magnitude is at most 6.

  attn    softmax(q K^T / sqrt(head_dim)) V over the positions below the sequence's length that have a page
  hold    rows of new K and V go to their positions' slots, quantised, and are read back as the values that are held
  rope    pairs of dims of q and k are rotated by their position times a frequency of the pair: (i, i + d / 2), or (2 i, 2 i + 1), of the
          first d dims of a head. `inverse` turns them back, which is the gradient's way
  tables  sequences get new lengths: pages are taken from a ring of free ones, first in first out, or given back to it, and the new
          positions are listed with their slots; then the lengths change back

Where `own` is true the library's entry points are called, otherwise the same is computed with elementary torch operations.

    python -c "from perf import more_operators; print(more_operators.listed())"
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp32": 4}
_LOWEST, _HIGHEST = -110, 126            # exponents of the scales
_CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _cached(name, kind, batch, q_heads, kv_heads, seq_len, rows, page, dtype="bf16", head_dim=128, ragged=False, holes=0.0):
    return {"name": name, "kind": kind, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "seq_len": seq_len, "rows": rows, "page": page, "dtype": dtype, "ragged": ragged, "holes": holes}


def _rope(name, rows, q_heads, k_heads, far, head_dim=128, rot_dim=128, interleaved=False, scaling="none", factor=1.0, theta=10000.0, dtype="bf16",
          inverse=False, fused=True):
    return {"name": name, "kind": "rope", "rows": rows, "q_heads": q_heads, "k_heads": k_heads, "far": far, "head_dim": head_dim,
            "rot_dim": rot_dim, "interleaved": interleaved, "scaling": scaling, "factor": factor, "theta": theta, "dtype": dtype,
            "inverse": inverse, "fused": fused}


def _tables(name, batch, longest, grow, page, holes=0.0, short=False):
    return {"name": name, "kind": "tables", "batch": batch, "longest": longest, "grow": grow, "page": page, "holes": holes, "short": short}


def listed():
    return [
        # one new token of one sequence: the smallest call of a decode loop, nothing but latency
        _cached("attn_one_token", "attn", 1, 32, 32, 512, 1, 16),
        # two long documents: few (sequence, head) pairs, so the length has to be split
        _cached("attn_one_token_long", "attn", 2, 28, 4, 131072, 1, 128),
        # a full batch of decoding sequences, the largest stream of keys and values
        _cached("attn_one_token_batch", "attn", 32, 32, 32, 4096, 1, 64, ragged=True),
        # active sets of different sizes, grouped-query heads, sizes that divide nothing, some pages given back
        _cached("attn_active_rows_ragged", "attn", 16, 28, 4, 769, 129, 32, ragged=True, holes=0.1),
        # a refresh of long sequences: every row attends to every position, bound by arithmetic
        _cached("attn_refresh", "attn", 4, 32, 32, 1536, 1536, 64),
        # what one denoising step writes
        _cached("hold_step", "hold", 8, 32, 32, 1024, 8, 16),
        # prompts written at once, and read back to hand them on
        _cached("hold_prompt", "hold", 4, 32, 32, 1536, 1536, 64),
        # the active rows of one denoising step, parts of the fused projection's rows
        _rope("rope_step", 64, 32, 32, 1024),
        # prompts at once
        _rope("rope_prompt", 6144, 32, 32, 1536),
        # long contexts, scaled by parts, interleaved pairs of half a head, grouped-query heads, fp32, back through a training step
        _rope("rope_long_gradient", 4099, 28, 4, 131072, rot_dim=64, interleaved=True, scaling="parts", factor=16.0, theta=500000.0, dtype="fp32",
              inverse=True, fused=False),
        # one block of new positions for each sequence of a batch, some sequences leave
        _tables("tables_step", 64, 4096, 32, 16, holes=0.05),
        # a queue of prompts is admitted at once, more than there are pages for
        _tables("tables_prompts", 512, 8192, 8192, 16, short=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


def draw(rng):
    """One more case of the ranges above (no name)."""
    while True:
        kind = rng.choice(("attn", "attn", "attn", "attn", "hold", "hold", "rope", "rope", "tables", "tables"))
        dtype, head_dim = "bf16", rng.choice((128, 128, 128, 64))
        q_heads, kv_heads = rng.choice(((32, 32), (32, 32), (28, 4), (24, 8), (16, 1)))
        if rng.random() < 0.2:
            dtype, head_dim, q_heads, kv_heads = "fp32", rng.choice((32, 64, 128)), 8, rng.choice((2, 8))
        if kind == "tables":
            longest = _log_int(rng, 1, 32768)
            c = _tables("", _log_int(rng, 1, 1024), longest, _log_int(rng, 1, longest), rng.choice((16, 32, 64, 256)), rng.choice((0.0, 0.0, 0.1)),
                        rng.random() < 0.3)
            if c["batch"] * longest > 512 * 8192:
                continue
        elif kind == "rope":
            rot = rng.choice((head_dim, head_dim, head_dim // 2, head_dim // 4, head_dim - 8, 10))
            scaling = rng.choice(("none", "none", "linear", "base", "parts"))
            c = _rope("", _log_int(rng, 1, 6144), q_heads, kv_heads, _log_int(rng, 64, 1 << 20), head_dim, rot, rng.random() < 0.5, scaling,
                      1.0 if scaling == "none" else rng.choice((2.0, 4.0, 16.0)), rng.choice((10000.0, 500000.0)), dtype, rng.random() < 0.3,
                      rng.random() < 0.5)
        else:
            seq_len = _log_int(rng, 1, 131072)
            rows = 1 if kind == "attn" and rng.random() < 0.4 else _log_int(rng, 1, min(seq_len, 1536))
            c = _cached("", kind, _log_int(rng, 1, 32), q_heads, kv_heads, seq_len, rows, rng.choice((16, 32, 64, 128, 256)), dtype, head_dim,
                        rng.random() < 0.5, rng.choice((0.0, 0.0, 0.1)))
            cells = c["batch"] * kv_heads * seq_len * head_dim
            scores = c["batch"] * q_heads * rows * seq_len
            if cells > 32 * 32 * 4096 * 128 or scores > 3.1e8 or (dtype == "fp32" and scores * head_dim > 5e9) or work(c)["bytes"] > 3e8:
                continue
        del c["name"]
        return c


# ---- the cache in 4 bits ----
def _lengths(case):
    """Keys and rows of each sequence; ragged: from all of them down to a few."""
    B, L, R = case["batch"], case["seq_len"], case["rows"]
    share = [(B - b) / B if case["ragged"] else 1.0 for b in range(B)]
    keys = [max(1, math.ceil(L * s)) for s in share]
    return keys, [min(k, max(1, math.ceil(R * s))) for k, s in zip(keys, share)]


def _quantise(x):
    """fp32 rows [..., n] -> (bytes of two codes [..., n / 2], biased exponents of the scales [..., n / 32])."""
    x = x.unflatten(-1, (-1, 32))
    m, up = torch.frexp(torch.where(torch.isfinite(x), x, 0.0).abs().amax(-1))             # m 2^up, m in [1/2, 1); 6 = 0.75 * 2^3
    e = torch.where(m > 0, up.to(torch.int32) - 3 + (m > 0.75).to(torch.int32), _LOWEST).clamp(_LOWEST, _HIGHEST)
    a = x.abs() * ((127 - e) << 23).view(torch.float32)[..., None]
    a = torch.where((e == _HIGHEST)[..., None], a.clamp(max=3.0), a)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    code = (code | torch.signbit(x).to(torch.uint8) << 3).flatten(-2)
    scale = torch.where(torch.isfinite(x).all(-1), e + 127, 255).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, scale


def _held(codes, scale):
    """The values that bytes of codes and scales stand for, in fp32."""
    table = torch.tensor([s * c for s in (1.0, -1.0) for c in _CODES], device=codes.device)
    x = table[torch.stack((codes & 15, codes >> 4), -1).to(torch.int32)].flatten(-2).unflatten(-1, (-1, 32))
    power = torch.where(scale == 255, float("nan"), (scale.to(torch.int32) << 23).view(torch.float32))
    return (x * power[..., None]).flatten(-2)


def _prepare_cache(case, seed, g):
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
    s = {"page_table": table, "seq_len": torch.tensor(keys, dtype=torch.int32, device="cuda")}
    for x in "kv":           # some dims are larger than others, as a projection's are
        s[x + "_pages"], s[x + "_scale"] = _quantise(normal(n_pages, Hkv, S, dh) * (0.5 + torch.rand((Hkv, 1, dh), generator=g, device="cuda")))
    # slots behind a sequence's end hold whatever was there before, here NaN
    tail = torch.tensor([k % S for k in keys], device="cuda")
    last = torch.gather(table, 1, needed - 1)[:, 0]
    for b in [b for b in range(B) if keys[b] % S and int(last[b]) >= 0]:
        for x in "kv":
            s[x + "_scale"][last[b], :, int(tail[b]):] = 255
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
    s["k"], s["v"] = normal(R, Hkv, dh).to(act), (2.0 * normal(R, Hkv, dh)).to(act)
    s["k_held"], s["v_held"] = (torch.zeros((R, Hkv, dh), dtype=act, device="cuda") for _ in range(2))
    return s


def _sequence_of_rows(s):
    return torch.searchsorted(s["row_off"][1:].contiguous(), torch.arange(s["rows"], device="cuda", dtype=torch.int32), right=True)


def _hold(s):
    S = s["k_pages"].shape[2]
    pos = s["pos"].long()
    page = s["page_table"][_sequence_of_rows(s), pos // S].long()
    there = (page >= 0) & (page < s["k_pages"].shape[0])
    page, slot = torch.where(there, page, 0), pos % S

    def one(new, pages, scale, out):
        codes, e = _quantise(new.float())
        at = page[there], slice(None), slot[there]
        pages[at], scale[at] = codes[there], e[there]
        out.copy_(torch.where(there[:, None, None], _held(pages[page, :, slot], scale[page, :, slot]), 0.0).to(out.dtype))

    one(s["k"], s["k_pages"], s["k_scale"], s["k_held"])
    one(s["v"], s["v_pages"], s["v_scale"], s["v_held"])


def _attend(s):
    q, table, off = s["q"], s["page_table"], s["row_off"].long()
    n_pages, Hkv, S, half = s["k_pages"].shape
    dh = 2 * half
    R, Hq = q.shape[:2]
    B, width = table.shape
    there = (table >= 0) & (table < n_pages)
    at = torch.where(there, table, 0).long()
    seen = there.repeat_interleave(S, dim=1, output_size=width * S) & (torch.arange(width * S, device="cuda")[None, :] < s["seq_len"][:, None])

    def gathered(pages, scale):                      # [B, Hkv, keys, dh] in fp32, zeros where nothing is seen
        x = _held(pages[at], scale[at]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, width * S, dh)
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


# ---- rotary positions ----
_ORIGINAL, _SLOW, _FAST = 4096, 1.0, 32.0          # scaled by parts: positions of the unscaled model; full turns over them


def _frequencies(case):
    """(radians of each pair for one position, in 64 bits, size of what comes out)."""
    d, theta, f = case["rot_dim"], case["theta"], case["factor"]
    if case["scaling"] == "base":
        theta = theta * f ** (d / (d - 2))
    freq = theta ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    if case["scaling"] == "linear":
        freq = freq / f
    if case["scaling"] == "parts":                 # pairs that turn often stay, those that hardly turn are stretched
        stay = ((_ORIGINAL * freq / (2.0 * math.pi) - _SLOW) / (_FAST - _SLOW)).clamp(0.0, 1.0)
        freq = freq * stay + freq / f * (1.0 - stay)
        return freq, 0.1 * math.log(f) + 1.0
    return freq, 1.0


def _prepare_rope(case, seed, g):
    R, Hq, Hk, dh = (case[k] for k in ("rows", "q_heads", "k_heads", "head_dim"))
    act = _TYPES[case["dtype"]]

    def normal(heads):
        return torch.randn((R, heads, dh), generator=g, device="cuda").to(act)

    if case["fused"]:
        qkv = normal(Hq + 2 * Hk)
        q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    else:
        q, k = normal(Hq), normal(Hk)
    freq, size = _frequencies(case)
    return {"q": q, "k": k, "pos": torch.randint(0, case["far"], (R,), generator=g, device="cuda", dtype=torch.int32), "case": case,
            "freq": freq.cuda(), "size": size, "q_out": torch.zeros((R, Hq, dh), dtype=act, device="cuda"),
            "k_out": torch.zeros((R, Hk, dh), dtype=act, device="cuda")}


def _rotate(s):
    d, half = s["case"]["rot_dim"], s["case"]["rot_dim"] // 2
    turn = s["pos"].double()[:, None] * s["freq"][None, :]
    cos = (torch.cos(turn) * s["size"]).float()[:, None, :]
    sin = (torch.sin(turn) * (-s["size"] if s["case"]["inverse"] else s["size"])).float()[:, None, :]

    def one(x, out):
        y = x.float()
        if s["case"]["interleaved"]:
            a, b = y[..., 0:d:2], y[..., 1:d:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = y[..., :half], y[..., half:d]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        out.copy_(torch.cat((turned, y[..., d:]), -1).to(out.dtype))

    one(s["q"], s["q_out"])
    one(s["k"], s["k_out"])


# ---- page tables ----
def _two_lengths(case):
    """Length of each sequence before and after."""
    B, top, grow = case["batch"], case["longest"], case["grow"]
    after = [max(1, math.ceil(top * (B - b) / B)) for b in range(B)]
    before = [max(0, n - 1 - 7 * b % B * (grow - 1) // B) if grow < top else 0 for b, n in enumerate(after)]
    leave = [b % 16 == 15 for b in range(B)]
    return [a if gone else n for n, a, gone in zip(before, after, leave)], [0 if gone else a for a, gone in zip(after, leave)]


def _prepare_tables(case, seed, g):
    B, S = case["batch"], case["page"]
    before, after = _two_lengths(case)
    order = torch.randperm(B, generator=torch.Generator().manual_seed(seed)).tolist()
    before, after = [before[i] for i in order], [after[i] for i in order]
    have, need = [-(-n // S) for n in before], [-(-n // S) for n in after]
    width = max(max(have), max(need)) + 1
    n_pages = sum(have) + (sum(max(0, y - x) for x, y in zip(have, need)) + 2) * (9 if case["short"] else 10) // 10 + 1
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    place, held = torch.arange(width, device="cuda")[None, :], torch.tensor(have, device="cuda")[:, None]
    first = torch.tensor([sum(have[:b]) for b in range(B)], device="cuda")[:, None]
    table = torch.where(place < held, ids[torch.where(place < held, first + place, 0)], -1)
    table = torch.where(torch.rand((B, width), generator=g, device="cuda") < case["holes"], -1, table).to(torch.int32).contiguous()
    # the free pages somewhere in the ring
    count, head = n_pages - sum(have), int(torch.randint(0, n_pages, (), generator=g, device="cuda"))
    ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(count, device="cuda")) % n_pages] = ids[sum(have):]
    s = {"page_table": table, "free_pages": ring, "page": S, "free_at": torch.tensor([head, count], dtype=torch.int32, device="cuda"),
         "seq_len": torch.tensor(before, dtype=torch.int32, device="cuda")}
    for name, x, y in (("there", before, after), ("back", after, before)):
        R = max(1, sum(max(0, b - a) for a, b in zip(x, y)))
        s[name] = {"lengths": torch.tensor(y, dtype=torch.int32, device="cuda"), "row_off": torch.zeros(B + 1, dtype=torch.int32, device="cuda"),
                   "pos": torch.full((R,), -1, dtype=torch.int32, device="cuda"), "slots": torch.full((R,), -1, dtype=torch.int64, device="cuda")}
    s["workspace"] = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    return s


def _resize(s, call):
    """Lengths in the order of the sequences: those that shrink give pages back, those that grow get pages until the first for which the
    free ones (before this call) or the rows of the lists do not last. A length below zero or beyond the table changes nothing."""
    table, ring, S, want = s["page_table"], s["free_pages"], s["page"], call["lengths"].long()
    B, width = table.shape
    N, R = ring.shape[0], call["pos"].shape[0]
    head, count = s["free_at"][0].long(), s["free_at"][1].long()
    old = s["seq_len"].long()
    new = torch.where((want < 0) | (want > width * S), old, want)
    have, need = (old + S - 1) // S, (new + S - 1) // S
    pages, rows = (need - have).clamp(min=0), (new - old).clamp(min=0)
    fits = (pages.cumsum(0) <= count) & (rows.cumsum(0) <= R)
    new = torch.where((new > old) & ~fits, old, new)
    need = (new + S - 1) // S
    pages, rows = (need - have).clamp(min=0), (new - old).clamp(min=0)
    # entries that get a page, and those that give theirs back: the first behind the ring's head, the others behind its end
    place = torch.arange(width, device="cuda")[None, :]
    gets, leaves = (place >= have[:, None]) & (place < need[:, None]), (place >= need[:, None]) & (place < have[:, None])
    given = (leaves & (table >= 0) & (table < N)).flatten()
    take = (pages.cumsum(0) - pages)[:, None] + place - have[:, None]
    taken = ring[(head + torch.where(gets, take, 0)) % N]
    spot = torch.where(given, (head + count + given.cumsum(0) - 1) % N, N)
    ring.copy_(torch.cat((ring, ring[:1])).scatter(0, spot, table.flatten())[:N])
    table.copy_(torch.where(gets, taken, torch.where(leaves, -1, table)))
    s["free_at"].copy_(torch.stack(((head + pages.sum()) % N, count - pages.sum() + given.sum())))
    s["seq_len"].copy_(new)
    call["row_off"][1:] = rows.cumsum(0)
    # the new positions and their slots
    off, r = call["row_off"].long(), torch.arange(R, device="cuda")
    seq = torch.searchsorted(off[1:].contiguous(), r, right=True).clamp(max=B - 1)
    p = old[seq] + r - off[seq]
    mine = r < off[-1]
    page = table[seq, torch.where(mine, p // S, 0)].long()
    slot = torch.where((page >= 0) & (page < N), page * S + p % S, -1)
    call["pos"].copy_(torch.where(mine, p, call["pos"].long()))
    call["slots"].copy_(torch.where(mine, slot, call["slots"]))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = {"rope": _prepare_rope, "tables": _prepare_tables}.get(case["kind"], _prepare_cache)
    return make(case, seed, g) | {"kind": case["kind"]}


def _library_rope(case):
    import paper_2505_15781_amd as P
    return P.Rope(case["head_dim"], case["rot_dim"], case["theta"], case["interleaved"], case["scaling"], case["factor"], _ORIGINAL, _SLOW, _FAST)


def _own(s):
    import paper_2505_15781_amd as P
    if s["kind"] == "rope":
        if "rope" not in s:                    # the frequencies of a model, made once
            s["rope"] = _library_rope(s["case"])
        P.rope(s["rope"], s["q"], s["k"], s["pos"], q_out=s["q_out"], k_out=s["k_out"], inverse=s["case"]["inverse"])
    elif s["kind"] == "tables":
        tables = P.PagedTables(s["page_table"], s["seq_len"], s["free_pages"], s["free_at"], s["page"])
        P.paged_resize(tables, s["there"]["lengths"], s["workspace"], s["there"]["row_off"], s["there"]["pos"], s["there"]["slots"])
        P.paged_resize(tables, s["back"]["lengths"], s["workspace"], s["back"]["row_off"], s["back"]["pos"], s["back"]["slots"])
    else:
        four, eight = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
        cache = P.PagedCache(s["k_pages"].view(four), s["v_pages"].view(four), s["page_table"], s["seq_len"], s["k_scale"].view(eight),
                             s["v_scale"].view(eight))
        if s["kind"] == "attn":
            P.paged_attn(cache, s["q"], s["row_off"], s["out"], s["max_rows"], s["workspace"])
        else:
            P.paged_store(cache, s["k"], s["v"], s["pos"], s["row_off"])
            P.paged_load(cache, s["k_held"], s["v_held"], s["pos"], s["row_off"])


def run(state):
    s = state
    if own:
        _own(s)
    elif s["kind"] == "tables":
        _resize(s, s["there"])
        _resize(s, s["back"])
    else:
        {"attn": _attend, "hold": _hold, "rope": _rotate}[s["kind"]](s)
    if s["kind"] == "attn":
        return {"out": s["out"]}
    if s["kind"] == "hold":
        return {"k_held": s["k_held"], "v_held": s["v_held"]}
    if s["kind"] == "rope":
        return {"q_out": s["q_out"], "k_out": s["k_out"]}
    return {k: s[k] for k in ("page_table", "seq_len", "free_pages", "free_at")} | {
        call + "_" + k: s[call][k] for call in ("there", "back") for k in ("row_off", "pos", "slots")}


def work(case):
    if case["kind"] == "tables":
        before, after = _two_lengths(case)
        S = case["page"]
        rows = sum(abs(x - y) for x, y in zip(before, after))                       # listed on the way there or back
        pages = sum(abs(-(-x // S) + y // -S) for x, y in zip(before, after))       # taken once and given back once
        return {"bytes": 12.0 * rows + 20.0 * pages + 2 * 16.0 * case["batch"], "flops": 0.0}
    es, dh = _BYTES[case["dtype"]], case["head_dim"]
    if case["kind"] == "rope":
        heads = case["q_heads"] + case["k_heads"]
        return {"bytes": case["rows"] * (2.0 * heads * dh * es + 4.0), "flops": 3.0 * case["rows"] * heads * case["rot_dim"]}
    keys, counts = _lengths(case)
    Hq, Hkv = case["q_heads"], case["kv_heads"]
    held = 2.0 * Hkv * (dh // 2 + dh // 32)                                          # K and V of a position
    if case["kind"] == "attn":
        return {"bytes": held * sum(keys) * (1.0 - case["holes"]) + 2.0 * sum(counts) * Hq * dh * es,
                "flops": sum(4.0 * Hq * dh * k * r for k, r in zip(keys, counts)) * (1.0 - case["holes"])}
    rows = sum(counts) * (1.0 - case["holes"])
    return {"bytes": 2.0 * rows * (held + 2.0 * Hkv * dh * es + 4.0), "flops": 4.0 * rows * Hkv * dh}


def exact(case, seed):
    """The same from the definitions in 64 bits; nothing for whole numbers."""
    s = prepare(case, seed)
    if case["kind"] == "tables":
        return None
    if case["kind"] == "rope":
        d, dh = case["rot_dim"], case["head_dim"]
        i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
        base = case["theta"] * (case["factor"] ** (d / (d - 2.0)) if case["scaling"] == "base" else 1.0)
        freq, size = torch.exp(-2.0 * i / d * math.log(base)), 1.0
        if case["scaling"] == "linear":
            freq /= case["factor"]
        elif case["scaling"] == "parts":
            share = torch.clamp((_ORIGINAL / (2.0 * math.pi / freq) - _SLOW) / (_FAST - _SLOW), 0.0, 1.0)
            freq = (1.0 - share) * (freq / case["factor"]) + share * freq
            size = 1.0 + 0.1 * math.log(case["factor"])
        angle = s["pos"].double()[:, None] * freq * (-1.0 if case["inverse"] else 1.0)
        turn = torch.polar(torch.full_like(angle, size), angle)[:, None, :]
        first = 2 * torch.arange(d // 2, device="cuda") if case["interleaved"] else torch.arange(d // 2, device="cuda")
        second = first + (1 if case["interleaved"] else d // 2)
        got = {}
        for x in "qk":
            y = s[x].double()
            z = torch.complex(y[..., first], y[..., second]) * turn
            out = y.clone()
            out[..., first], out[..., second] = z.real, z.imag
            got[x + "_out"] = out
        return got
    n_pages, Hkv, S, half = s["k_pages"].shape
    dh = 2 * half
    table, off, keys = s["page_table"].tolist(), s["row_off"].tolist(), s["seq_len"].tolist()
    value = torch.tensor([(-1.0 if c & 8 else 1.0) * ((c & 1) * 0.5 if c & 7 < 2 else (1.0 + (c & 1) * 0.5) * 2.0 ** ((c & 7) // 2 - 1))
                          for c in range(16)], dtype=torch.float64, device="cuda")

    def values(pages, scale, ids):                   # [Hkv, len(ids) * S, dh]
        x, power = pages[ids].long(), torch.exp2(scale[ids].double() - 127.0).repeat_interleave(32, dim=-1)
        both = torch.empty((*x.shape[:-1], dh), dtype=torch.float64, device="cuda")
        both[..., 0::2], both[..., 1::2] = value[x % 16], value[x // 16]
        return (both * power).transpose(0, 1).reshape(Hkv, -1, dh)

    if case["kind"] == "attn":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        group = case["q_heads"] // Hkv
        for b, n in enumerate(keys):
            held = [(j, p) for j, p in enumerate(table[b]) if 0 <= p < n_pages and j * S < n]
            if not held:
                continue
            at = (torch.tensor([j for j, _ in held], device="cuda")[:, None] * S + torch.arange(S, device="cuda")).reshape(-1)
            ids = torch.tensor([p for _, p in held], device="cuda")
            k, v = (values(s[x + "_pages"], s[x + "_scale"], ids)[:, at < n] for x in "kv")
            for h in range(case["q_heads"]):
                z = s["q"][off[b]:off[b + 1], h].double() @ k[h // group].T.contiguous() / math.sqrt(dh)
                out[off[b]:off[b + 1], h] = torch.softmax(z, dim=-1) @ v[h // group]
        return {"out": out}
    pos = s["pos"].long()
    seq = torch.repeat_interleave(torch.arange(len(keys), device="cuda"), torch.diff(s["row_off"]).long())
    page = s["page_table"].long()[seq, torch.div(pos, S, rounding_mode="floor")]
    there = ((page >= 0) & (page < n_pages))[:, None, None]
    got = {}
    for x in "kv":
        y = s[x].double().unflatten(-1, (-1, 32))
        e = torch.ceil(torch.log2(y.abs().amax(-1, keepdim=True).clamp(min=1e-300) / 6.0)).clamp(-110, 126)
        z = y / torch.exp2(e)
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=1.0))) - 1)       # distance of neighbouring e2m1 values
        got[x + "_held"] = torch.where(there, (torch.round(z / step) * step * torch.exp2(e)).flatten(-2), 0.0)
    return got
