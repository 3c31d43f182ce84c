"""The operators beside the verification step, as cases to measure: what draws the drafts, what extends and moves the paths of a
sequence, and what keeps the pages of their cache in line.  One pass = one call through `paper_2511_15898_amd.binding`, or, with
`own` false, the same results from elementary torch operations.

A case is a dict of plain values:
  op      "draft"    gr_draft_logits / gr_draft: n i.i.d. drafts per row, top-k or whole row
          "select"   gr_beam_select: the M best continuations of the K beams of each of S sequences
          "reorder"  gr_beam_reorder: the beams' states follow their parents, in place, dense or by block table
          "pages"    gr_page_update: block tables, slot maps and the free list after lengths have changed
  dtype   of the logits, or of the state
  pad     (draft, select) elements between the end of a row and the beginning of the next: a padded output projection
Rows stand in for language models' next-token distributions: heavy-tailed logits, as in `workloads.py`."""
import math
import weakref

import torch

own = False

ROW_OK, ROW_BAD, ROW_NO_ROOM = 0, 3, 4


def _draft(name, rows, B, V, n, k, dtype="float32", pad=0):
    return {"name": name, "op": "draft", "rows": rows, "B": B, "V": V, "n": n, "k": k, "dtype": dtype, "pad": pad, "t_lo": 0.6, "t_hi": 1.4}


def _select(name, S, K, V, M, dtype="float32", pad=0, done=0.0, warm=False):
    return {"name": name, "op": "select", "S": S, "K": K, "V": V, "M": M, "dtype": dtype, "pad": pad, "done": done, "warm": warm}


def _reorder(name, layout, O, S, K, H, T, D, block, lo, hi, shared, dtype="bfloat16"):
    return {"name": name, "op": "reorder", "layout": layout, "O": O, "S": S, "K": K, "H": H, "T": T, "D": D, "block": block, "lo": lo, "hi": hi,
            "shared": shared, "dtype": dtype}


def _pages(name, R, block, width, lo, hi, grow_lo, grow_hi, shrink=0.0, spare=1.5):
    return {"name": name, "op": "pages", "R": R, "block": block, "width": width, "lo": lo, "hi": hi, "grow_lo": grow_lo, "grow_hi": grow_hi,
            "shrink": shrink, "spare": spare}


def listed():
    return [
        # one sequence: its four drafts out of one row of draft logits
        _draft("draft, one row", "logits", 1, 32000, 4, 64),
        # the verifier's large configuration: eight drafts a row, top-k 128, as a 16-bit draft model leaves its logits
        _draft("draft, large vocabulary", "logits", 256, 128256, 8, 128, dtype="bfloat16"),
        # no top-k, probabilities, sizes that are multiples of nothing
        _draft("draft, whole rows", "probs", 203, 50021, 16, 0),
        # one sequence, four beams
        _select("beams of one sequence", 1, 4, 32000, 4),
        # an ordinary batch, twice as many candidates as beams (some will end), 16-bit logits, temperatures
        _select("beams of a batch", 32, 8, 128256, 16, dtype="bfloat16", done=0.1, warm=True),
        # many sequences, ten beams, rows of a padded projection
        _select("beams, many and wide", 64, 10, 128256, 20, pad=64),
        # one sequence's attention states in one dense buffer, head by head
        _reorder("states of one sequence", "heads", 8, 1, 4, 8, 512, 64, 0, 200, 400, 0.0),
        # a batch's pages: the prompt's are shared by the beams, what was generated is moved
        _reorder("states in pages", "paged", 8, 16, 4, 8, 1024, 128, 16, 300, 1000, 0.5),
        # the states of a recurrent model: no tokens, whole rows
        _reorder("whole states", "whole", 24, 16, 8, 1, 1, 65536, 0, 1, 1, 0.0, dtype="float32"),
        # a decoding step: a token to each request
        _pages("pages, one token each", 64, 16, 512, 100, 4000, 1, 1),
        # after a verification: up to nine tokens more, some sequences end and give all back
        _pages("pages after a verification", 4096, 16, 256, 0, 3900, 0, 9, shrink=0.1),
        # prompts come in
        _pages("pages of new prompts", 512, 64, 128, 0, 0, 1, 4096),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["draft", "select", "reorder", "pages"])
    if kind == "draft":
        B, V = _log_between(rng, 1, 512), _log_between(rng, 300, 128256)
        rows = rng.choice(["logits", "logits", "probs"])
        case = _draft("", rows, min(B, (1 << 25) // V), V, rng.randint(1, 16), rng.choice([0, _log_between(rng, 1, 256), _log_between(rng, 1, 256)]),
                      dtype=rng.choice(["float32", "bfloat16", "float16"]) if rows == "logits" else "float32", pad=rng.choice([0, 0, rng.randint(1, 64)]))
    elif kind == "select":
        K, V = rng.randint(1, 16), _log_between(rng, 100, 128256)
        S = max(1, min(_log_between(rng, 1, 128), (1 << 26) // (K * V)))
        M = min(rng.choice([K, 2 * K, rng.randint(1, 64)]), 64)
        case = _select("", S, K, V, M, dtype=rng.choice(["float32", "bfloat16", "float16"]), pad=rng.choice([0, 0, rng.randint(1, 64)]),
                       done=rng.choice([0.0, 0.0, 0.3]), warm=rng.random() < 0.5)
    elif kind == "reorder":
        layout = rng.choice(["heads", "tokens", "paged", "paged", "whole"])
        dtype = rng.choice(["bfloat16", "float32", "float16", "uint8"])
        O, K, H = _log_between(rng, 1, 32), rng.randint(2, 16), rng.randint(1, 16)
        T, D = (1, _log_between(rng, 64, 100000)) if layout == "whole" else (_log_between(rng, 16, 4000), rng.choice([64, 80, 96, 128, rng.randint(16, 256)]))
        H = 1 if layout == "whole" else H
        S = max(1, min(_log_between(rng, 1, 32), (1 << 28) // (O * K * H * T * D)))
        O = max(1, min(O, (1 << 28) // (S * K * H * T * D)))
        lo = rng.randint(0, T) if T > 1 else 1
        case = _reorder("", layout, O, S, K, H, T, D, rng.choice([8, 16, 16, 32, 64, 13]) if layout == "paged" else 0, lo, T,
                        rng.choice([0.0, 0.3, 0.8]) if T > 1 else 0.0, dtype=dtype)
    else:
        R, block = _log_between(rng, 1, 4096), rng.choice([1, 8, 16, 16, 32, 64, 128, 13])
        hi = _log_between(rng, 16, 4000)
        grow = rng.choice([1, rng.randint(1, 16), _log_between(rng, 1, max(2, min(4096, 1000000 // R)))])
        width = (hi + grow + block - 1) // block + rng.randint(0, 8)
        lo = rng.randint(0, hi)
        case = _pages("", R, block, width, lo, hi, rng.randint(0, grow), grow, shrink=rng.choice([0.0, 0.1, 0.5]), spare=rng.choice([1.5, 1.5, 0.4]))
    del case["name"]
    return case


class _State:
    pass


def _spread(count, lo, hi, gen):
    """`count` whole numbers spread evenly from lo to hi, in an order of the seed's: sums and sizes are the same for every seed."""
    even = lo + torch.arange(count, device="cuda") * (hi - lo) // max(1, count - 1)
    return even[torch.randperm(count, device="cuda", generator=gen)].int()


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _heavy_rows(rows, V, pad, gen):
    """Heavy-tailed logits 4 * Gumbel(0, 1), float32, [rows, V] within rows of V + pad."""
    wide = torch.empty((rows, V + pad), device="cuda").exponential_(generator=gen).clamp_(min=1e-9).log_().mul_(-4.0)
    return wide


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = _generator(seed)
    return {"draft": _prepare_draft, "select": _prepare_select, "reorder": _prepare_reorder, "pages": _prepare_pages}[case["op"]](s, case, gen)


def _prepare_draft(s, c, gen):
    B, V = c["B"], c["V"]
    wide = _heavy_rows(B, V, c["pad"], gen)
    s.temperature = torch.empty(B, device="cuda").uniform_(c["t_lo"], c["t_hi"], generator=gen)
    if c["rows"] == "probs":
        wide[:, :V] = torch.softmax(wide[:, :V] / s.temperature[:, None], 1)
    s.x = wide.to(getattr(torch, c["dtype"]))[:, :V]
    s.uniforms = torch.rand((B, c["n"]), device="cuda", generator=gen).clamp_(max=1.0 - 2.0 ** -24)
    s.drafts = torch.empty((B, c["n"]), dtype=torch.int32, device="cuda")
    s.status = torch.empty(B, dtype=torch.int32, device="cuda")
    return s


def _prepare_select(s, c, gen):
    S, K, V, M = c["S"], c["K"], c["V"], c["M"]
    s.logits = _heavy_rows(S * K, V, c["pad"], gen).to(getattr(torch, c["dtype"])).view(S, K, V + c["pad"])[:, :, :V]
    # running sums of log probabilities of beams that are some tokens long; the last beam of a few sequences is not in use
    s.scores = torch.empty((S, K), device="cuda").uniform_(-25.0, -15.0, generator=gen).sort(1, descending=True)[0]
    if K > 1:
        s.scores[::5, K - 1] = -math.inf
    s.temperature = torch.empty(S, device="cuda").uniform_(0.7, 1.3, generator=gen) if c["warm"] else None
    s.finished, s.eos = None, -1
    if c["done"]:
        s.finished = (torch.rand((S, K), device="cuda", generator=gen) < c["done"]).to(torch.uint8)
        s.eos = min(2, V - 1)
    s.out = (torch.empty((S, M), device="cuda"), torch.empty((S, M), dtype=torch.int32, device="cuda"), torch.empty((S, M), dtype=torch.int32, device="cuda"),
             torch.empty((S, M), dtype=torch.uint8, device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda"))
    return s


def _random_state(shape, dtype, gen):
    if dtype == "uint8":
        return torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=gen)
    return torch.empty(shape, dtype=getattr(torch, dtype), device="cuda").uniform_(-1.0, 1.0, generator=gen)


def _prepare_reorder(s, c, gen):
    O, S, K, H, T, D = (c[w] for w in ("O", "S", "K", "H", "T", "D"))
    s.parent = torch.randint(0, K, (S, K), dtype=torch.int32, device="cuda", generator=gen)
    s.first = s.length = s.table = None
    if c["layout"] != "whole":
        s.length = _spread(S, c["lo"], c["hi"], gen)
        s.first = (s.length * c["shared"]).int()
    if c["layout"] == "paged":
        bs = c["block"]
        width = (T + bs - 1) // bs
        j = torch.arange(width, device="cuda")[None, None, :]
        used = (j < ((s.length + bs - 1) // bs)[:, None, None]).expand(S, K, width)
        common = (j < (s.first // bs)[:, None, None]).expand(S, K, width)           # the prompt's pages: those of beam 0
        own_page = used & (~common | (torch.arange(K, device="cuda")[None, :, None] == 0))
        count = int(own_page.sum())
        blocks = count + 3
        table = torch.full((S, K, width), -1, dtype=torch.int32, device="cuda")
        table[own_page] = torch.randperm(blocks, device="cuda", generator=gen)[:count].int()
        s.table = torch.where(common, table[:, :1], table).reshape(S * K, width).contiguous()
        s.state = _random_state((O, blocks, H, bs, D), c["dtype"], gen)
    elif c["layout"] == "tokens":
        s.state = _random_state((O, S * K, T, H, D), c["dtype"], gen).transpose(2, 3)
    else:
        s.state = _random_state((O, S * K, H, T, D), c["dtype"], gen)
    return s


def _prepare_pages(s, c, gen):
    R, bs, width = c["R"], c["block"], c["width"]
    s.lengths = _spread(R, c["lo"], c["hi"], gen)
    grown = torch.minimum(s.lengths + _spread(R, c["grow_lo"], c["grow_hi"], gen), torch.tensor(width * bs, dtype=torch.int32, device="cuda"))
    back = torch.rand(R, device="cuda", generator=gen) < c["shrink"]
    s.new_lengths = torch.where(back, (s.lengths * torch.randint(0, 2, (R,), device="cuda", generator=gen) * 0.9).int(), grown)
    s.table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    held = torch.arange(width, device="cuda")[None, :] < ((s.lengths + bs - 1) // bs)[:, None]
    need = int(((s.new_lengths + bs - 1) // bs - (s.lengths + bs - 1) // bs).clamp(min=0).sum())
    taken = int(held.sum())
    spare = int(need * c["spare"]) + 1
    pool = R * ((c["hi"] + bs - 1) // bs + 2 * ((c["grow_hi"] + bs - 1) // bs + 1)) + 1      # all blocks: more than are held and asked for
    ids = torch.randperm(pool, device="cuda", generator=gen).int()
    s.table[held] = ids[:taken]
    s.free_blocks = torch.full((pool,), -1, dtype=torch.int32, device="cuda")
    s.free_blocks[:spare] = ids[taken:taken + spare]
    s.free_count = torch.tensor([spare], dtype=torch.int32, device="cuda")
    s.slots = torch.full((R * c["grow_hi"] + 5,), -7, dtype=torch.int64, device="cuda")
    s.out = (torch.empty(R, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda"),
             torch.empty(R + 1, dtype=torch.int32, device="cuda"), torch.empty(R, dtype=torch.int32, device="cuda"))
    return s


# ---------------------------------------------------------------- the plain forms

def _plain_draft(s):
    c = s.case
    V, k = c["V"], c["k"] if 0 < c["k"] < c["V"] else c["V"]
    x = s.x.float()
    ids = None
    if k < V:
        ids = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k].sort(1)[0]
        x = x.gather(1, ids)
    x = x.double()                                                    # a draw stands next to a border of the distribution
    if c["rows"] == "logits":
        x = torch.exp((x - x.amax(1, keepdim=True)) / s.temperature.double()[:, None])
    mass = x.cumsum(1)
    at = torch.searchsorted(mass, s.uniforms.double() * mass[:, -1:], right=True).clamp(max=k - 1)
    return (at if ids is None else ids.gather(1, at)).int(), torch.zeros_like(s.status)


def _plain_select(s):
    c = s.case
    S, K, V, M = c["S"], c["K"], c["V"], c["M"]
    x = s.logits.double()                                             # beams meet at borders that float32 sums would blur
    if s.temperature is not None:
        x = x / s.temperature.double()[:, None, None]
    top = x.amax(2, keepdim=True)
    x = s.scores.double()[:, :, None] + (x - top - torch.log(torch.exp(x - top).sum(2, keepdim=True)))
    if s.finished is not None:
        done = (s.finished != 0)[:, :, None]
        at_end = (torch.arange(V, device="cuda") == s.eos)[None, None, :]
        x = torch.where(done, torch.where(at_end, s.scores.double()[:, :, None], -math.inf), x)
    value, index = torch.sort(x.view(S, K * V), dim=1, descending=True, stable=True)
    value, index = value[:, :M], index[:, :M]
    if M > K * V:
        value = torch.nn.functional.pad(value, (0, M - K * V), value=-math.inf)
        index = torch.nn.functional.pad(index, (0, M - K * V))
    none = value == -math.inf
    parent = torch.where(none, -1, index // V).int()
    token = torch.where(none, -1, index % V).int()
    over = ~none & (token == s.eos) if s.eos >= 0 else torch.zeros_like(none)
    return value.float(), parent, token, over.to(torch.uint8), torch.zeros(S, dtype=torch.int32, device="cuda")


def _plain_reorder(s):
    c = s.case
    S, K, T, bs = c["S"], c["K"], c["T"], c["block"]
    rows = torch.arange(S * K, device="cuda")
    source = (rows // K) * K + s.parent.view(-1).long()
    if c["layout"] == "whole":
        s.state.copy_(s.state[:, source])
        return s.state
    t = torch.arange(T, device="cuda")
    moved = ((t[None, :] >= s.first[:, None]) & (t[None, :] < s.length[:, None])).repeat_interleave(K, 0) & (source != rows)[:, None]
    if c["layout"] != "paged":
        s.state.copy_(torch.where(moved[None, :, None, :, None], s.state[:, source], s.state))
        return s.state
    to, t = moved.nonzero(as_tuple=True)
    page, old, at = s.table[to, t // bs].long(), s.table[source[to], t // bs].long(), t % bs
    s.state[:, page, :, at] = s.state[:, old, :, at]
    return s.state


def _plain_pages(s):
    c = s.case
    bs, width = c["block"], c["width"]
    old, new = s.lengths.long(), s.new_lengths.long()
    had, has = (old + bs - 1) // bs, (new + bs - 1) // bs
    need, more = (has - had).clamp(min=0), (new - old).clamp(min=0)
    count = s.free_count.long()
    have = count + (had - has).clamp(min=0).sum()
    ok = (new <= old) | ((need.cumsum(0) <= have) & (more.cumsum(0) <= s.slots.numel()))
    left = have - (need * ok).sum()
    j = torch.arange(width, device="cuda")[None, :]
    released = s.table[(j >= has[:, None]) & (j < had[:, None])]
    stack = s.free_blocks.clone()
    stack[count + torch.arange(released.numel(), device="cuda")] = released
    grown = (j >= had[:, None]) & (j < has[:, None]) & ok[:, None]
    s.table[grown] = stack[have - 1 - torch.arange(int(grown.sum()), device="cuda")]
    at = torch.arange(stack.numel(), device="cuda")
    s.free_blocks.copy_(torch.where((at >= count) & (at < left), stack, s.free_blocks))
    starts = torch.nn.functional.pad((more * ok).cumsum(0), (1, 0))
    t = torch.arange(s.slots.numel(), device="cuda")
    r = torch.searchsorted(starts[1:], t, right=True).clamp(max=old.numel() - 1)
    position = (old[r] + t - starts[r]).clamp(min=0, max=width * bs - 1)
    slot = s.table[r, position // bs].long() * bs + position % bs
    s.slots.copy_(torch.where(t < starts[-1], slot, s.slots))
    return (torch.where(ok, new, old).int(), left.int(), starts.int(), torch.where(ok, ROW_OK, ROW_NO_ROOM).int(), s.slots, s.table, s.free_blocks)


# ---------------------------------------------------------------- the framework's calls

def _handle(s, rows):
    """The handle that a program creates once for its rows."""
    if not hasattr(s, "handle"):
        from paper_2511_15898_amd import binding as gr
        s.handle = gr.gr_create(rows, s.case["V"])
        weakref.finalize(s, gr.gr_destroy, s.handle)
    return s.handle


def _own_draft(s):
    from paper_2511_15898_amd import binding as gr
    c = s.case
    h = _handle(s, c["B"])
    if c["rows"] == "probs":
        return gr.gr_draft(h, s.x, c["n"], c["k"], s.uniforms, s.drafts, s.status)
    return gr.gr_draft_logits(h, s.x, s.temperature, c["n"], c["k"], s.uniforms, s.drafts, s.status)


def _own_select(s):
    from paper_2511_15898_amd import binding as gr
    c = s.case
    return gr.gr_beam_select(_handle(s, c["S"] * c["K"]), s.logits, s.scores, c["M"], temperature=s.temperature, finished=s.finished, eos=s.eos, out=s.out)


def _own_reorder(s):
    from paper_2511_15898_amd import binding as gr
    return gr.gr_beam_reorder(s.state, s.parent, s.first, s.length, s.table)


def _own_pages(s):
    from paper_2511_15898_amd import binding as gr
    out = gr.gr_page_update(s.lengths, s.new_lengths, s.table, s.free_blocks, s.free_count, s.case["block"], s.slots, s.out)
    return (*out, s.slots, s.table, s.free_blocks)


def run(s):
    op = s.case["op"]
    if own:
        return {"draft": _own_draft, "select": _own_select, "reorder": _own_reorder, "pages": _own_pages}[op](s)
    return {"draft": _plain_draft, "select": _plain_select, "reorder": _plain_reorder, "pages": _plain_pages}[op](s)


def exact(case, seed):
    """The scores of a selection, from the definition; everything else that is returned is whole numbers or copies."""
    if case["op"] != "select":
        return None
    s = prepare(case, seed)
    S, K, M = case["S"], case["K"], case["M"]
    best = []
    for b in range(K):                                                # a beam at a time, its M largest at most
        z = s.logits[:, b].to(torch.float64)
        if s.temperature is not None:
            z = z / s.temperature.to(torch.float64).unsqueeze(1)
        z = torch.log_softmax(z, dim=1).topk(min(M, case["V"]), dim=1).values + s.scores[:, b, None].to(torch.float64)
        if s.finished is not None:
            alone = torch.full_like(z, -math.inf)
            alone[:, 0] = s.scores[:, b].to(torch.float64)
            z = torch.where(s.finished[:, b, None] != 0, alone, z)
        best.append(z)
    best = torch.cat(best + [torch.full((S, M), -math.inf, dtype=torch.float64, device="cuda")], 1)
    return best.topk(M, dim=1).values, None, None, None, None


_SIZE = {"float32": 4, "bfloat16": 2, "float16": 2, "uint8": 1}


def work(case):
    """Bytes: what is read and written once, lengths and choices of parents taken at their means.  Operations: a comparison for
    every element of a row, and where its sum is asked for an exponential (about 16 operations) and an addition."""
    c = case
    if c["op"] == "draft":
        rows = c["B"] * c["V"]
        return {"bytes": rows * _SIZE[c["dtype"]] + c["B"] * (8 * c["n"] + 8), "flops": rows * (17 if c["rows"] == "logits" and not 0 < c["k"] < c["V"] else 2)}
    if c["op"] == "select":
        rows = c["S"] * c["K"] * c["V"] * (1.0 - c["done"])
        return {"bytes": rows * _SIZE[c["dtype"]] + 5 * c["S"] * c["K"] + 13 * c["S"] * c["M"], "flops": rows * 18}
    if c["op"] == "reorder":
        K = c["K"]
        written = 1.0 - 1.0 / K                                       # beams whose parent is another
        read = 1.0 - (1.0 - 1.0 / K) ** (K - 1)                       # beams that another one takes
        tokens = 0.5 * (c["lo"] + c["hi"]) * (1.0 - c["shared"])
        return {"bytes": c["O"] * c["S"] * K * c["H"] * c["D"] * _SIZE[c["dtype"]] * tokens * (read + written) + 4 * c["S"] * K, "flops": 0}
    grow = 0.5 * (c["grow_lo"] + c["grow_hi"]) * (1.0 - c["shrink"])
    blocks = grow / c["block"] + c["shrink"] * 0.5 * (c["lo"] + c["hi"]) * 0.55 / c["block"]
    return {"bytes": c["R"] * (24 + 8 * grow + 8 * blocks), "flops": 0}
