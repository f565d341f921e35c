"""Attention whose keys are not its queries' own tokens, and the paged 8-bit cache that holds such keys, as measurable cases.

Four operators, each as a user's program calls it, and in its plain form in 32-bit torch arithmetic:

  append   K and V of a call's tokens go behind what their sequences hold in a paged cache of e4m3 codes with one scale per page and
           head.  A page that gets a larger value has its codes re-expressed under the larger scale.
  attend   the queries of one token or of a chunk attend to everything that their sequences hold in that cache; "step" appends the
           call's own K and V first.
  cross    the tokens of a clip attend to an encoder's states: another length, ragged or masked.
  pages    pages are copied, sequences forked (full pages shared, the last one copied) and freed, the pool compacted.

Keys of a case: `op`, and
  append, attend, step   B sequences, Hq query heads, H cached heads, d, page, N (tokens that the longest sequence holds after the call), T (tokens
           of the call per sequence), ragged (sequences and calls of different lengths), causal, tokens_first ([B, T, H, d] in memory)
  cross    B, Hq, H, N queries, S keys, d, keys ("all", "lengths", "mask"), tokens_first
  pages    do ("copy", "fork", "compact"), form (the cache's format), H, d, page, rows (sequences), N (tokens of the longest sequence),
           forks (sequences that are freed and take over another's tokens), n (pages copied)
"""
import math

import torch

own = False


def listed():
    cache = dict(d=128, page=64, ragged=False, causal=False, tokens_first=True)
    cross = dict(op="cross", d=128, keys="lengths", tokens_first=True)
    pages = dict(op="pages", form="e4m3_page", d=128, page=64, forks=0, n=0)
    return [
        # one new token of 64 sequences, somewhere in their last pages: latency
        dict(cache, name="append_token", op="append", B=64, Hq=8, H=8, N=2049, T=1, ragged=True),
        # K and V of a whole clip behind a first frame that does not end with a page
        dict(cache, name="append_clip", op="append", B=1, Hq=24, H=24, N=32767, T=32750),
        # one token of a short sequence is appended and attends: the smallest call
        dict(cache, name="step_one_token", op="step", B=1, Hq=16, H=16, N=255, T=1),
        # one token of eight long sequences, grouped heads: the cache's bytes are the work
        dict(cache, name="attend_long_grouped", op="attend", B=8, Hq=32, H=8, N=131071, T=1, ragged=True),
        # prompts of odd sizes behind a shared prefix, token by token causal, grouped heads of 64
        dict(cache, name="attend_prompt_causal", op="attend", B=3, Hq=32, H=8, d=64, page=48, N=8190, T=777, ragged=True, causal=True),
        # three frames of a clip that is generated in chunks attend to all 32 760 tokens; the largest
        dict(cache, name="step_chunk_of_clip", op="step", B=1, Hq=24, H=24, N=32760, T=4680),
        # a single query token per item of a guidance pair to a short prompt: latency
        dict(cross, name="cross_one_token", B=2, Hq=16, H=16, N=1, S=77, d=64),
        # a guidance pair of the 32 760-token clip to two prompts of 512 places
        dict(cross, name="cross_clip_text", B=2, Hq=24, H=24, N=32760, S=512),
        # a long encoder sequence with places masked out among the others, grouped heads, sizes that divide nothing
        dict(cross, name="cross_masked_long", B=1, Hq=32, H=8, N=8191, S=4095, keys="mask", tokens_first=False),
        # half of 64 hypotheses are dropped and replaced by copies of the better half
        dict(pages, name="pages_fork", do="fork", H=8, rows=64, N=4000, forks=32),
        # sequences have come and gone: the pool's live pages move to its front
        dict(pages, name="pages_compact", do="compact", H=24, rows=12, N=9000),
        # a few pages of a cache with a scale per token are copied: latency
        dict(pages, name="pages_copy", do="copy", form="e4m3", H=16, rows=4, N=1000, n=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: single tokens to the largest chunk, short to long caches, odd sizes, every option."""
    op = rng.choice(("append", "attend", "step", "cross", "cross", "pages"))
    d = rng.choice((64, 128, 128))
    if op == "pages":
        do, form = rng.choice(("copy", "fork", "compact")), rng.choice(("e4m3_page", "e4m3_page", "e4m3", "fp4"))
        while True:
            H, page, rows, N = _log_int(rng, 1, 32), rng.choice((16, 48, 64, 128)), rng.randint(2, 96), _log_int(rng, 1, 16384)
            if rows * N * H * d <= 400_000_000:
                break
        return dict(op=op, do=do, form=form, H=H, d=d, page=page, rows=rows, N=N, forks=rng.randint(1, rows // 2) if do == "fork" else 0,
                    n=_log_int(rng, 1, max(1, rows * (-(-N // page)) // 2)) if do == "copy" else 0)
    tokens_first, group = rng.random() < 0.5, rng.choice((1, 1, 2, 4, 7))
    if op == "cross":
        while True:
            B, H, N, S = rng.choice((1, 1, 2, 3)), _log_int(rng, 1, 32), _log_int(rng, 1, 32760), _log_int(rng, 1, 8192)
            if rng.random() < 0.2:
                B, N = _log_int(rng, 1, 32), rng.choice((1, 1, 2, 5))
            if B * H * group * N * d <= 2 * 24 * 32760 * 128 and B * H * group * N * S * d <= 8191 * 4095 * 32 * 128 and B * H * S * d <= 40_000_000:
                break
        return dict(op=op, B=B, Hq=H * group, H=H, N=N, S=S, d=d, keys=rng.choice(("all", "lengths", "lengths", "mask")), tokens_first=tokens_first)
    while True:
        B, H, N = rng.choice((1, 1, 2, 3, 8)), _log_int(rng, 1, 24), _log_int(rng, 1, 131072)
        T = rng.choice((1, 1, _log_int(rng, 1, 128), _log_int(rng, 1, 8192)))
        if rng.random() < 0.2:
            B, T = _log_int(rng, 1, 64), 1
        if T <= N and B * H * N * d <= 1_100_000_000 and B * H * group * T * d <= 40_000_000 and (
                op == "append" or B * H * group * T * N * d <= 24 * 4680 * 32760 * 128):
            break
    return dict(op=op, B=B, Hq=H * group, H=H, d=d, page=rng.choice((16, 48, 64, 64, 128)), N=N, T=T, ragged=rng.random() < 0.5,
                causal=op != "append" and rng.random() < 0.4, tokens_first=tokens_first)


def work(case):
    d, H = case["d"], case["H"]
    if case["op"] == "cross":
        q = case["B"] * case["Hq"] * case["N"] * d
        there = 1.0 if case["keys"] == "all" else 0.75                                  # of the keys, on average
        return {"bytes": 4.0 * q + 4.0 * case["B"] * H * case["S"] * d * there, "flops": 4.0 * q * case["S"] * there}
    if case["op"] == "pages":
        held = {"e4m3_page": d, "e4m3": d + 4, "fp4": d // 2 + d // 16 + 4}[case["form"]]
        page = 2.0 * H * (case["page"] * held + 4 * (case["form"] == "e4m3_page"))
        per = -(-case["N"] // case["page"])
        # (compaction: 30 % of the pages are free, and about that part of the others lies behind the border)
        moved = {"copy": case["n"], "fork": case["forks"], "compact": 0.21 * per * case["rows"]}[case["do"]]
        return {"bytes": 2.0 * moved * page + 8.0 * per * case["rows"], "flops": 0.0}
    ragged = 0.75 if case["ragged"] else 1.0
    new, keys = case["B"] * case["T"] * ragged, case["B"] * case["N"] * ragged
    total, flops = 0.0, 0.0
    if case["op"] != "attend":
        total += 2 * H * new * (2 * d + d)
    if case["op"] != "append":
        total += 2 * H * keys * d + 4 * case["Hq"] * new * d + 4 * case["Hq"] * new
        seen = case["N"] * ragged - (0.5 * case["T"] * ragged if case["causal"] else 0.0)
        flops = 4.0 * case["Hq"] * new * seen * d
    return {"bytes": float(total), "flops": float(flops)}


class State:
    pass


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _heads(gen, B, H, N, d, tokens_first):
    """[B, H, N, d], or the same as a view of [B, N, H, d]."""
    x = torch.randn(B, N, H, d, generator=gen, device="cuda", dtype=torch.bfloat16) if tokens_first else \
        torch.randn(B, H, N, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    return x.transpose(1, 2) if tokens_first else x


def _quotient(a, b):
    """a / b with b a number, divided rather than multiplied by its reciprocal."""
    return a / torch.full((), b, dtype=a.dtype, device=a.device)


def _e4m3(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _codes_under(x, scale):
    """e4m3 codes (bytes) of fp32 x under a scale that is broadcast against it; zeros where it is 0."""
    there = scale != 0
    return _e4m3(torch.where(there, x / torch.where(there, scale, torch.ones_like(scale)), torch.zeros_like(x))).view(torch.uint8)


def _randint(gen, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=gen, device="cuda")


# ---------------------------------------------------------------------------------------------------------- states
def prepare(case, seed):
    s, gen = State(), _generator(seed)
    s.case, s.plan, s.cache_plan = case, None, None
    {"cross": _prepare_cross, "pages": _prepare_pages}.get(case["op"], _prepare_cache)(s, case, gen)
    return s


def _prepare_cache(s, case, gen):
    B, Hq, H, d, page, N, T = (case[n] for n in ("B", "Hq", "H", "d", "page", "N", "T"))
    per = -(-N // page)
    pages = B * per + 3
    s.table = torch.randperm(pages, generator=gen, device="cuda")[:B * per].view(B, per).to(torch.int32).contiguous()
    s.counts = torch.full((B,), T, dtype=torch.int32, device="cuda")
    after = torch.full((B,), N, dtype=torch.int32, device="cuda")
    if case["ragged"]:
        s.counts = _randint(gen, max(1, T // 2), T, B).to(torch.int32)
        after = torch.maximum(_randint(gen, max(1, N // 2), N, B).to(torch.int32), s.counts)
    s.after, s.before = after, after - s.counts
    s.k = []                                                                         # codes and scales of K, then of V
    for arrays in range(2):
        codes, scale = [], []
        for h in range(H):                                                           # (a head at a time: less memory at once)
            x = torch.randn(pages, page, d, generator=gen, device="cuda") * torch.exp(0.3 * torch.randn(pages, 1, 1, generator=gen, device="cuda"))
            top = _quotient(x.to(torch.bfloat16).float().abs().amax((1, 2)), 448.0)
            codes.append(_codes_under(x.to(torch.bfloat16).float(), top[:, None, None]))
            scale.append(top)
        s.k.append([torch.stack(codes, 1), torch.stack(scale, 1).contiguous()])
    s.k, s.v = s.k
    if case["op"] != "attend":
        s.new_k, s.new_v = (_heads(gen, B, H, T, d, case["tokens_first"]) for _ in range(2))
    if case["op"] != "append":
        s.q = _heads(gen, B, Hq, T, d, case["tokens_first"])
        s.o = torch.zeros_like(s.q)                                                  # (rows behind a sequence's last query stay as they are)
        s.lse = torch.zeros(B, Hq, T, dtype=torch.float32, device="cuda")


def _prepare_cross(s, case, gen):
    B, Hq, H, N, S, d = (case[n] for n in ("B", "Hq", "H", "N", "S", "d"))
    s.q = _heads(gen, B, Hq, N, d, case["tokens_first"])
    s.k, s.v = (_heads(gen, B, H, S, d, case["tokens_first"]) for _ in range(2))
    s.o = torch.empty_like(s.q)
    s.lengths = _randint(gen, max(1, S // 2), S, B).to(torch.int32) if case["keys"] == "lengths" else None
    s.mask = None
    if case["keys"] == "mask":
        s.mask = torch.rand(B, S, generator=gen, device="cuda") < 0.75
        s.mask[:, 0] = True


def _prepare_pages(s, case, gen):
    H, d, page, rows, N = (case[n] for n in ("H", "d", "page", "rows", "N"))
    per = -(-N // page)
    live = rows * per
    spare = max(live * 3 // 7, case["forks"] + 1)                                    # 30 % of the pool is free
    pages = live + spare
    s.pages = pages
    s.k, s.v = [], []
    for arrays in (s.k, s.v):
        # (any byte but the two NaNs is a code; scales as a normal distribution gives them)
        row = d // 2 if case["form"] == "fp4" else d
        codes = torch.randint(0, 127, (pages, H, page, row), generator=gen, device="cuda", dtype=torch.uint8)
        codes += (torch.randint(0, 2, (pages, H, page, row), generator=gen, device="cuda", dtype=torch.uint8) << 7)
        arrays.append(codes)
        arrays.append((torch.rand(*((pages, H) if case["form"] == "e4m3_page" else (pages, H, page)), generator=gen, device="cuda") + 0.5) / 112)
        if case["form"] == "fp4":
            arrays.append(torch.randint(1, 127, (pages, H, page, d // 16), generator=gen, device="cuda", dtype=torch.uint8))
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    if case["do"] == "copy":
        s.src, s.dst = order[:case["n"]].contiguous(), order[case["n"]:2 * case["n"]].contiguous()
        return
    s.lengths0 = _randint(gen, max(1, N // 2), N, rows).to(torch.int32)
    s.table0 = order[:live].view(rows, per).clone()
    used = (s.lengths0 + page - 1) // page
    s.table0[torch.arange(per, device="cuda")[None] >= used[:, None]] = -1
    s.refs0 = torch.zeros(pages, dtype=torch.int32, device="cuda")
    s.refs0[s.table0[s.table0 >= 0].long()] = 1
    if case["do"] == "fork":
        who = torch.randperm(rows, generator=gen, device="cuda").to(torch.int32)
        s.children = who[:case["forks"]].contiguous()
        s.parents = who[case["forks"]:][_randint(gen, 0, rows - case["forks"] - 1, case["forks"])].contiguous()
        s.keep = torch.zeros(case["forks"], dtype=torch.int32, device="cuda")
    s.table, s.lengths, s.refs = s.table0.clone(), s.lengths0.clone(), s.refs0.clone()
    s.work = torch.empty(8 * pages + 256, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"cross": _cross, "pages": _pages}.get(s.case["op"], _cached)(s)


def _append(arrays, x, s):
    """Plain form of the append: the pages that a call touches, old rows beside new ones."""
    codes, scale = arrays
    B, H, T, d = x.shape
    page = s.case["page"]
    first = s.before.long() // page
    touched = first[:, None] + torch.arange((T - 1) // page + 2, device="cuda")                      # [B, P]
    place = touched[..., None] * page + torch.arange(page, device="cuda")                            # [B, P, page]
    t = place - s.before[:, None, None]
    new, old = (t >= 0) & (t < s.counts[:, None, None]), t < 0
    b, p = torch.nonzero(new.any(-1), as_tuple=True)                                                 # pages with something new
    ids = s.table[b, touched[b, p]].long()
    new, old, t = new[b, p], old[b, p], t[b, p].clamp(0, T - 1)
    rows = x.transpose(1, 2)[b[:, None], t].float().transpose(1, 2)                                  # [pages, H, page, d]
    rows = torch.where(new[:, None, :, None], rows, torch.zeros_like(rows))
    held, held_scale = codes[ids], torch.where(old.any(-1)[:, None], scale[ids], torch.zeros_like(scale[ids]))
    top = torch.maximum(held_scale, _quotient(rows.abs().amax((2, 3)), 448.0))
    ratio = torch.where(top != 0, held_scale / torch.where(top != 0, top, torch.ones_like(top)), torch.zeros_like(top))
    again = _e4m3(held.view(torch.float8_e4m3fn).float() * ratio[..., None, None]).view(torch.uint8)
    again = torch.where((top > held_scale)[..., None, None], again, held)
    fresh = _codes_under(rows, top[..., None, None])
    new, old = new[:, None, :, None], old[:, None, :, None]
    codes[ids] = torch.where(new, fresh, torch.where(old, again, held))
    scale[ids] = top


def _softmax_rows(q, k, v, there, scale):
    """q [.., T, d], k and v [.., N, d], there [T, N] or [1, N]: softmax(q k^T) v and the log-sum-exp; zeros and -inf where nothing is there."""
    logits = torch.where(there, (q @ k.mT) * scale, torch.full((), -math.inf, dtype=q.dtype, device=q.device))
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return o, (torch.log(total) + top)[..., 0]


def _attention(q, keys, there, B, Hq, H, T, N, d, dtype):
    """As many heads and queries at a time as memory likes; keys(b, heads) gives K and V [heads, N, d], there(b, t0, t1) what may be seen."""
    o = torch.zeros(B, Hq, T, d, dtype=dtype, device="cuda")
    lse = torch.zeros(B, Hq, T, dtype=dtype, device="cuda")
    group, scale = Hq // H, 1.0 / math.sqrt(d)
    heads = max(1, min(H, (1 << 28) // (N * group * T)))
    step = max(1, (1 << 28) // (N * group * heads))
    for b in range(B):
        for h0 in range(0, H, heads):
            h1 = min(H, h0 + heads)
            k, v = keys(b, slice(h0, h1))
            mine = slice(h0 * group, h1 * group)
            for t0 in range(0, T, step):
                t1 = min(T, t0 + step)
                rows = q[b, mine, t0:t1].to(dtype).unflatten(0, (h1 - h0, group))
                got, total = _softmax_rows(rows, k[:, None], v[:, None], there(b, t0, t1), scale)
                o[b, mine, t0:t1], lse[b, mine, t0:t1] = got.flatten(0, 1), total.flatten(0, 1)
    return o, lse


def _cached(s):
    c = s.case
    if own:
        from paper_2606_23743_b200 import binding as sva
        if s.cache_plan is None:
            s.cache_plan = sva.make_kv_cache(s.k, s.v, "e4m3_page")
        if c["op"] != "attend":
            sva.kv_cache_append(s.cache_plan, s.new_k, s.new_v, s.table, s.before, s.counts)
        if c["op"] != "append":
            if s.plan is None:
                s.plan = sva.make_cached_attn(s.cache_plan, s.q, s.o, s.table, causal=c["causal"])
                s.workspace = torch.empty(sva.cached_attn_workspace_bytes(s.plan), dtype=torch.uint8, device="cuda")
            sva.cached_attn_fwd(s.plan, s.q, s.table, s.after, s.o, s.counts, s.lse, workspace=s.workspace)
    else:
        if c["op"] != "attend":
            _append(s.k, s.new_k, s)
            _append(s.v, s.new_v, s)
        if c["op"] != "append":
            B, Hq, H, d, T = c["B"], c["Hq"], c["H"], c["d"], c["T"]
            N = s.table.shape[1] * c["page"]
            place, t = torch.arange(N, device="cuda"), torch.arange(T, device="cuda")

            def keys(b, heads):
                ids = s.table[b].long()
                return [(a[0][ids, heads].view(torch.float8_e4m3fn).float() * a[1][ids, heads][..., None, None]).transpose(0, 1).flatten(1, 2)
                        for a in (s.k, s.v)]

            def there(b, t0, t1):
                end = (s.before[b] + t[t0:t1] + 1 if c["causal"] else s.after[b].expand(t1 - t0))[:, None]
                return place[None] < end

            o, lse = _attention(s.q, keys, there, B, Hq, H, T, N, d, torch.float32)
            query = t[None, None] < s.counts[:, None, None]
            s.o = torch.where(query[..., None], o, torch.zeros_like(o)).to(torch.bfloat16)
            s.lse = torch.where(query, lse, torch.zeros_like(lse))
    codes = (s.k[0].view(torch.float8_e4m3fn), s.k[1], s.v[0].view(torch.float8_e4m3fn), s.v[1])
    return codes if c["op"] == "append" else (s.o, s.lse) if c["op"] == "attend" else (s.o, s.lse) + codes


def _cross(s):
    c = s.case
    if own:
        from paper_2606_23743_b200 import binding as sva
        if s.plan is None:
            s.plan = sva.make_cross_attn(s.q, s.k, s.v, s.o)
            s.workspace = torch.empty(sva.cross_attn_workspace_bytes(s.plan), dtype=torch.uint8, device="cuda")
        sva.cross_attn_fwd(s.plan, s.q, s.k, s.v, s.o, s.lengths, s.mask, workspace=s.workspace)
        return s.o
    place = torch.arange(c["S"], device="cuda")

    def there(b, t0, t1):
        return s.mask[b][None] if s.mask is not None else (place < s.lengths[b])[None] if s.lengths is not None else (place >= 0)[None]

    return _attention(s.q, lambda b, h: (s.k[b, h].float(), s.v[b, h].float()), there, c["B"], c["Hq"], c["H"], c["N"], c["S"], c["d"],
                      torch.float32)[0].to(torch.bfloat16)


def _pages(s):
    c = s.case
    arrays = s.k + s.v
    page = c["page"]
    if own and s.cache_plan is None:
        from paper_2606_23743_b200 import binding as sva
        s.cache_plan = sva.make_kv_cache(s.k, s.v, c["form"])
    if c["do"] == "copy":
        if own:
            from paper_2606_23743_b200 import binding as sva
            sva.kv_pages_copy(s.cache_plan, s.src, s.dst)
        else:
            for a in arrays:
                a[s.dst.long()] = a[s.src.long()]
        return arrays
    # (the pool's state as it is before the call; the pages' contents are the same however often it is made)
    s.table.copy_(s.table0)
    s.lengths.copy_(s.lengths0)
    s.refs.copy_(s.refs0)
    if own:
        from paper_2606_23743_b200 import binding as sva
        if c["do"] == "fork":
            sva.kv_pages_free(s.cache_plan, s.refs, s.table, s.lengths, s.children, s.keep)
            sva.kv_pages_fork(s.cache_plan, s.refs, s.table, s.lengths, s.parents, s.children)
        else:
            sva.kv_pages_compact(s.cache_plan, s.refs, s.table, s.work)
    elif c["do"] == "fork":
        children, parents = s.children.long(), s.parents.long()
        column = torch.arange(s.table.shape[1], device="cuda")[None]
        rows = s.table[children]                                                     # freed: everything from place `keep` on
        gone = (column >= (s.keep[:, None] + page - 1) // page) & (rows >= 0)
        s.refs.index_add_(0, rows[gone].long(), torch.full((), -1, dtype=torch.int32, device="cuda").expand(int(gone.sum())))
        s.table[children] = torch.where(gone, torch.full_like(rows, -1), rows)
        s.lengths[children] = torch.minimum(s.lengths[children], s.keep)
        rows, length = s.table[parents], s.lengths[parents]                          # forked: full pages shared, the last one copied
        shared = column < (length // page)[:, None]
        partial = length % page > 0
        free = torch.sort((s.refs != 0).to(torch.int32), stable=True)[1]
        fresh = free[(torch.cumsum(partial, 0) - 1).clamp(min=0)][partial]
        held = rows[partial, (length // page)[partial].long()].long()
        for a in arrays:
            a[fresh] = a[held]
        rows = torch.where(shared, rows, torch.full_like(rows, -1))
        s.refs.index_add_(0, rows[shared].long(), torch.ones((), dtype=torch.int32, device="cuda").expand(int(shared.sum())))
        s.refs[fresh] = 1
        rows[partial, (length // page)[partial].long()] = fresh.to(torch.int32)
        s.table[children] = rows
        s.lengths[children] = length
    else:
        live = s.refs > 0
        ids = torch.arange(s.pages, device="cuda")
        border = live.sum()
        src, dst = ids[live & (ids >= border)], ids[~live & (ids < border)]
        for a in arrays:
            a[dst] = a[src]
        ids[src] = dst
        s.refs[dst] = s.refs[src]
        s.refs[src] = 0
        s.table.copy_(torch.where(s.table >= 0, ids[s.table.clamp(min=0).long()].to(torch.int32), s.table))
    return [s.table, s.lengths, s.refs] + arrays


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def _nearest_e4m3(y):
    """y rounded to the nearest e4m3 number, ties to even."""
    exponent = torch.frexp(y)[1].clamp(min=-5) - 1
    unit = torch.ldexp(torch.ones_like(y), exponent - 3)
    return (torch.round(y / unit) * unit).clamp(-448.0, 448.0)


def _as_fp32(y):
    return y.to(torch.float32).to(torch.float64)


def _exact_append(codes, scale, x, s):
    """Values of the codes, and scales, after the append: sequence by sequence and page by page.  Scales and quotients are fp32 numbers by definition."""
    page = s.case["page"]
    value, scale = codes.view(torch.float8_e4m3fn).double(), scale.double().clone()
    before, counts, table = s.before.tolist(), s.counts.tolist(), s.table.tolist()
    for b in range(s.case["B"]):
        at, end = before[b], before[b] + counts[b]
        while at < end:
            stop = min(end, (at // page + 1) * page)
            i, lo, hi = table[b][at // page], at % page, at % page + stop - at
            rows = x[b, :, at - before[b]:stop - before[b]].double()
            held = scale[i] if lo else torch.zeros_like(scale[i])
            top = torch.maximum(held, _as_fp32(rows.abs().amax((1, 2)) / 448.0))
            if lo:
                ratio = _as_fp32(held / top)[:, None, None]
                value[i, :, :lo] = torch.where((top > held)[:, None, None], _nearest_e4m3(_as_fp32(value[i, :, :lo] * ratio)), value[i, :, :lo])
            value[i, :, lo:hi] = _nearest_e4m3(_as_fp32(rows / top[:, None, None]))
            scale[i] = top
            at = stop
    return value, scale


def exact(case, seed):
    # (pages are moved as they are: nothing is computed.  Cases whose 64-bit arithmetic would take long are left out.)
    if case["op"] == "pages" or work(case)["flops"] > 1e13:
        return None
    s = prepare(case, seed)
    if case["op"] == "cross":
        there = torch.ones(case["B"], case["S"], dtype=torch.bool, device="cuda")
        if s.lengths is not None:
            there = torch.arange(case["S"], device="cuda")[None] < s.lengths[:, None]
        if s.mask is not None:
            there = s.mask
        return _exact_attention(s.q, lambda b, h: (s.k[b, h][there[b]].double(), s.v[b, h][there[b]].double(), None), case)[0]
    arrays = [(codes.view(torch.float8_e4m3fn), scale.double()) for codes, scale in (s.k, s.v)]
    if case["op"] != "attend":
        arrays = [_exact_append(a[0], a[1], x, s) for a, x in ((s.k, s.new_k), (s.v, s.new_v))]
    flat = (arrays[0][0].double(), arrays[0][1], arrays[1][0].double(), arrays[1][1]) if case["op"] != "attend" else ()
    if case["op"] == "append":
        return flat
    before, after, counts = s.before.tolist(), s.after.tolist(), s.counts.tolist()

    def keys(b, h):
        ids = s.table[b].long()
        k, v = ((a[0][ids, h].double() * a[1][ids, h][:, None, None]).flatten(0, 1)[:after[b]] for a in arrays)
        return k, v, before[b] if case["causal"] else None

    o, lse = _exact_attention(s.q, keys, case)
    for b in range(case["B"]):
        o[b, :, counts[b]:] = 0
        lse[b, :, counts[b]:] = 0
    return (o, lse) + flat


def _exact_attention(q, keys, case):
    """Per query head, in 64 bits, over the keys that are there; causal from the position that keys() gives on."""
    B, Hq, T, d = q.shape
    o, lse = torch.zeros(B, Hq, T, d, dtype=torch.float64, device="cuda"), torch.zeros(B, Hq, T, dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(case["H"]):
            k, v, first = keys(b, h)
            step = max(1, (1 << 26) // max(1, k.shape[0]))
            for head in range(h * (Hq // case["H"]), (h + 1) * (Hq // case["H"])):
                for t0 in range(0, T, step):
                    x = torch.einsum("td,nd->tn", q[b, head, t0:t0 + step].double(), k) * d ** -0.5
                    if first is not None:
                        n = torch.arange(k.shape[0], device="cuda")
                        x.masked_fill_(n[None] > first + torch.arange(t0, t0 + x.shape[0], device="cuda")[:, None], -math.inf)
                    lse[b, head, t0:t0 + step] = torch.logsumexp(x, -1)
                    o[b, head, t0:t0 + step] = torch.einsum("tn,nd->td", torch.exp(x - lse[b, head, t0:t0 + step, None]), v)
    return o, lse
