"""Timing cases of answering from a compacted cache: what a serving program has the library do after the compression pass.

Kinds of a case:
  append   the tokens of a step rotated to their positions and written into a paged cache (kvm_paged_append)
  attn     attention of the rows of a batch over the compacted cache of their prompt, shared by all rows of the prompt, and over
           each row's own paged tail (kvm_prefix_attn)
  step     one layer of a decoding step: both calls, one after the other

A prompt's compacted cache has as many states in a head as the merge left there, so the prefix lengths differ from head to head
and the rows beyond them are whatever the memory held.  Queries, keys and values are N(0, 1) as in the other timing cases.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HEAD_DIM = 128
ROPE_BASE = 10000.0


def _case(name, kind, P, B, T, H, G, cap, tail, page, dtype, rot=128, interleaved=0, ragged=0, far=0):
    return {"name": name, "kind": kind, "P": P, "B": B, "T": T, "H": H, "G": G, "cap": cap, "tail": tail, "page": page,
            "dtype": dtype, "rot": rot, "interleaved": interleaved, "ragged": ragged, "far": far}


def listed():
    return [
        # one token of one row, one layer of a 32-head model: nothing but launch and latency
        _case("append_f16_1x1_32", "append", 1, 1, 1, 32, 1, 0, 300, 16, "f16"),
        # one token of each row of a large batch, grouped queries
        _case("append_bf16_256x1_8g4", "append", 1, 256, 1, 8, 4, 0, 1000, 64, "bf16", ragged=1),
        # a few follow-up questions of different lengths, half of each head rotated, neighbouring pairs, far positions
        _case("append_f32_6x301_8g2_rot64", "append", 1, 6, 301, 8, 2, 0, 700, 32, "f32", rot=64, interleaved=1, ragged=1,
              far=1000000),
        # prompts of four rows appended whole, one layer of a 40-head model
        _case("append_f16_4x4096_40", "append", 1, 4, 4096, 40, 1, 0, 4096, 64, "f16"),
        # one row answers from the 4096-token prompt's cache at one half: the smallest call
        _case("attn_f16_1x1_32_c2048", "attn", 1, 1, 1, 32, 1, 2048, 100, 16, "f16"),
        # 64 answers sampled from one prompt of 16384 tokens, grouped queries
        _case("attn_bf16_64x1_8g4_c8192", "attn", 1, 64, 1, 8, 4, 8192, 512, 64, "bf16", ragged=1),
        # a running batch: four prompts with different numbers of rows, tails from one token on, small pages
        _case("attn_f16_37x1_32_c2048_ragged", "attn", 4, 37, 1, 32, 1, 2048, 1000, 16, "f16", ragged=1),
        # three drafted tokens a row checked at once, fp32
        _case("attn_f32_10x3_8g2_c1433", "attn", 2, 10, 3, 8, 2, 1433, 250, 32, "f32", ragged=1),
        # long answers, one for each of eight prompts: the tails are what is read
        _case("attn_f16_8x1_32_c5734_t16384", "attn", 8, 8, 1, 32, 1, 5734, 16384, 64, "f16", ragged=1),
        # follow-up questions of up to 1000 tokens over one long context
        _case("attn_bf16_4x1000_8g4_c8192", "attn", 1, 4, 1000, 8, 4, 8192, 1000, 64, "bf16", ragged=1),
        # the largest: two prompts, four rows each with 2048 new tokens, one layer of a 40-head model
        _case("attn_bf16_8x2048_40_c5734", "attn", 2, 8, 2048, 40, 1, 5734, 2048, 64, "bf16"),
        # one layer of a decoding step: 32 rows of two prompts
        _case("step_f16_32x1_32_c2048", "step", 2, 32, 1, 32, 1, 2048, 600, 32, "f16", ragged=1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "attn", "step"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    H, G = rng.choice([(1, 1), (4, 2), (8, 1), (8, 4), (8, 2), (16, 1), (32, 1), (40, 1), (4, 8)])
    T = rng.choice([1, 1, 1, _log(rng, 2, 8), _log(rng, 9, 2048)])
    if kind == "step" and T > 8:
        T = 1
    B = _log(rng, 1, 256 if T == 1 else (64 if T <= 8 else 8))
    P = _log(rng, 1, min(B, 8))
    cap = _log(rng, 64, 8192) if kind != "append" else 0
    tail = max(T, _log(rng, 1, 16384 if B <= 8 else 1024))
    # bounded by the work of the largest listed cases
    while B > 1 and B * T * H * G * (cap + tail) > 8 * 2048 * 40 * (5734 + 2048) // (8 if dtype == "f32" else 1):
        B = (B + 1) // 2
    while T > 1 and B * T * H * G * (cap + tail) > 8 * 2048 * 40 * (5734 + 2048) // (8 if dtype == "f32" else 1):
        T = (T + 1) // 2
    while B > 1 and kind == "append" and B * T * H * (G + 2) > 4 * 4096 * 40 * 3 // (2 if dtype == "f32" else 1):
        B = (B + 1) // 2
    while B > 1 and B * tail * H > 8 * 16384 * 32 // (2 if dtype == "f32" else 1):
        B = (B + 1) // 2
    P = min(P, B)
    rot = rng.choice([128, 128, 64, 32]) if kind != "attn" else 128
    return {"kind": kind, "P": P, "B": B, "T": T, "H": H, "G": G, "cap": cap, "tail": tail,
            "page": rng.choice([16, 16, 32, 64, 128]), "dtype": dtype, "rot": rot,
            "interleaved": rng.choice([0, 1]) if kind != "attn" else 0, "ragged": rng.choice([0, 1, 1]),
            "far": rng.choice([0, 0, 100000, 1000000]) if kind != "attn" else 0}


def _frac(i, step=0.6180339887):
    return (i * step + 0.31) % 1.0


def new_lengths(case):
    """New tokens of every row: T, or spread over one to T (the first row always T)."""
    B, T = case["B"], case["T"]
    if not case["ragged"] or T == 1:
        return [T] * B
    return [T if b == 0 else max(1, int(round(T * (0.3 + 0.7 * _frac(b))))) for b in range(B)]


def tail_lengths(case):
    """Tokens of every row's own tail once the new ones are in it."""
    new, tail = new_lengths(case), case["tail"]
    if not case["ragged"]:
        return [tail] * case["B"]
    return [tail if b == 0 else max(n, int(round(tail * _frac(b, 0.7548776662)))) for b, n in enumerate(new)]


def prefix_lengths(case):
    """States a head of a prompt's compacted cache holds."""
    P, H, cap = case["P"], case["H"], case["cap"]
    lens = [[max(1, int(cap * (0.62 + 0.38 * _frac(p * H + h)))) for h in range(H)] for p in range(P)]
    return np.array(lens, dtype=np.int32)


def row_starts(case):
    """Rows [start[p], start[p + 1]) belong to prompt p; every prompt has one at least."""
    P, B = case["P"], case["B"]
    if not case["ragged"] and B % P == 0:
        return [p * (B // P) for p in range(P + 1)]
    cuts = [0]
    for p in range(1, P):
        even = B * p // P
        cuts.append(min(max(cuts[-1] + 1, even + (p % 2) * (B // (3 * P))), B - (P - p)))
    return cuts + [B]


def _normal(gen, shape, dt):
    out = torch.empty(shape, dtype=dt, device="cuda")
    flat = out.view(-1)
    step = 1 << 27
    for i in range(0, flat.numel(), step):
        flat[i:i + step] = torch.randn((min(step, flat.numel() - i),), generator=gen, device="cuda").to(dt)
    return out


class State:
    pass


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind, P, B, T, H, G, cap = (case[k] for k in ("kind", "P", "B", "T", "H", "G", "cap"))
    dt, page = DTYPES[case["dtype"]], case["page"]
    i32 = dict(dtype=torch.int32, device="cuda")
    s = State()
    s.kind, s.H, s.G, s.rot, s.interleaved, s.page = kind, H, G, case["rot"], bool(case["interleaved"]), page
    new, tail = new_lengths(case), tail_lengths(case)
    s.new_lens = torch.tensor(new, **i32)
    # where the append writes the lengths, nothing that looks like them stands before the call
    s.kv_lens = torch.tensor(tail, **i32) if kind == "attn" else torch.full((B,), -1, **i32)
    s.past_lens = torch.tensor([t - n for t, n in zip(tail, new)], **i32)
    # the tails: pages scattered over a pool, entries behind a row's last page are not in use
    used = [-(-t // page) for t in tail]
    max_pages = max(used) + 1
    n_pages = sum(used) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    s.table = torch.full((B, max_pages), -1, **i32)
    at = 0
    for b in range(B):
        s.table[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
    s.K_pages = _normal(gen, (n_pages, H, page, HEAD_DIM), dt)
    s.V_pages = _normal(gen, (n_pages, H, page, HEAD_DIM), dt)
    qkv = _normal(gen, (B, T, (G + 2) * H, HEAD_DIM), dt)     # a fused projection's output, one row a token
    s.q, s.k, s.v = qkv[:, :, :G * H], qkv[:, :, G * H:(G + 1) * H], qkv[:, :, (G + 1) * H:]
    if kind == "attn":
        s.q = s.q.contiguous()                                # rotated queries as the append leaves them
    else:
        s.q_out = torch.zeros((B, T, G * H, HEAD_DIM), dtype=dt, device="cuda")
        s.inv_freq = (1.0 / ROPE_BASE ** (torch.arange(0, s.rot, 2, dtype=torch.float64) / max(s.rot, 1))).float().cuda()
        at = case["far"] if case["far"] else 2 * cap + 512
        s.pos_base = torch.tensor([max(0, at - 37 * b) for b in range(B)], **i32)
    if kind != "append":
        starts = row_starts(case)
        s.row_prefix = [p for p in range(P) for _ in range(starts[p], starts[p + 1])]
        even = all(starts[p] * P == p * B for p in range(P + 1))
        s.row_start = None if even else torch.tensor(starts, **i32)
        s.prefix_lens = torch.from_numpy(prefix_lengths(case)).cuda()
        s.K_pre = _normal(gen, (P, H, cap, HEAD_DIM), dt)
        s.V_pre = _normal(gen, (P, H, cap, HEAD_DIM), dt)
        s.out = torch.zeros((B, T, G * H, HEAD_DIM), dtype=dt, device="cuda")
        s.lse = torch.zeros((B, T, G * H), dtype=torch.float32, device="cuda") if kind == "attn" else None
    s.shape = None
    if own:
        _handles(s)
    return s


def _handles(s):
    from paper_2407_08454_amd import binding as kb
    s.kb = kb
    T = s.q.shape[1]
    s.pages = kb.make_pages(s.K_pages, s.V_pages, s.table)
    s.shape = kb.make_token_shape(s.pages, T, s.G, s.new_lens if T > 1 else None)
    if s.kind != "attn":
        s.rotation = kb.make_rotation(s.inv_freq, interleaved=s.interleaved)
    if s.kind != "append":
        s.prefix = kb.make_prefix(s.K_pre, s.V_pre, s.prefix_lens, s.row_start)
        s.ws = torch.empty(max(kb.kvm_prefix_attn_workspace_bytes(s.shape, s.prefix, s.pages), 256), dtype=torch.uint8,
                           device="cuda")


def run(s):
    if not own:
        return _plain(s)
    if s.shape is None:
        _handles(s)
    kb = s.kb
    outputs = []
    q = s.q
    if s.kind != "attn":
        kb.kvm_paged_append(s.shape, s.pages, s.rotation, s.q, s.k, s.v, s.past_lens, s.pos_base, s.q_out, s.kv_lens)
        outputs += [s.q_out, s.K_pages, s.V_pages, s.kv_lens]
        q = s.q_out
    if s.kind != "append":
        kb.kvm_prefix_attn(s.shape, s.prefix, s.pages, q, s.kv_lens, s.out, s.lse, s.ws)
        outputs += [s.out] if s.lse is None else [s.out, s.lse]
    return outputs


# ---- the plain forms ----------------------------------------------------------------------------------

def _plain(s):
    outputs = []
    q = s.q
    if s.kind != "attn":
        _plain_append(s)
        outputs += [s.q_out, s.K_pages, s.V_pages, s.kv_lens]
        q = s.q_out
    if s.kind != "append":
        _plain_attention(s, q)
        outputs += [s.out] if s.lse is None else [s.out, s.lse]
    return outputs


def _turn(x, cos, sin, rot, interleaved):
    x = x.float()
    out = x.clone()
    half = rot // 2
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :half], x[..., half:rot])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        out[..., 0:rot:2], out[..., 1:rot:2] = ra, rb
    else:
        out[..., :half], out[..., half:rot] = ra, rb
    return out


def _plain_append(s):
    B, T = s.q.shape[:2]
    dt = s.q.dtype
    t = torch.arange(T, device="cuda")
    slot = s.past_lens.long()[:, None] + t[None, :]
    valid = t[None, :] < s.new_lens.long()[:, None]
    angle = (s.pos_base.long()[:, None] + slot).double()[..., None] * s.inv_freq.double()
    cos, sin = torch.cos(angle).float()[:, :, None, :], torch.sin(angle).float()[:, :, None, :]
    q = _turn(s.q, cos, sin, s.rot, s.interleaved).to(dt)
    k = _turn(s.k, cos, sin, s.rot, s.interleaved).to(dt)
    s.q_out.copy_(torch.where(valid[:, :, None, None], q, s.q_out))
    rows, tokens = valid.nonzero(as_tuple=True)
    at = slot[rows, tokens]
    pages = s.table.long()[rows, at // s.page]
    s.K_pages[pages, :, at % s.page] = k[rows, tokens]
    s.V_pages[pages, :, at % s.page] = s.v[rows, tokens]
    s.kv_lens.copy_(s.past_lens + s.new_lens)


def _plain_attention(s, q):
    B, T, HG, d = q.shape
    H, G = s.H, s.G
    cap = s.K_pre.shape[2]
    dt = q.dtype
    t = torch.arange(T, device="cuda")
    slots = torch.arange(s.table.shape[1] * s.page, device="cuda")
    states = torch.arange(cap, device="cuda")
    heads = max(1, int(1.5e9 / (G * T * (cap + slots.numel()))))      # of one row at a time
    for b in range(B):
        p = s.row_prefix[b]
        pages = s.table[b].long().clamp(min=0)
        seen = slots[None, :] <= (s.kv_lens[b] - s.new_lens[b] + t)[:, None]             # (T, slots)
        valid = t < s.new_lens[b]
        for h in range(0, H, heads):
            n = min(heads, H - h)
            K = torch.cat([s.K_pre[p, h:h + n].float(), s.K_pages[pages, h:h + n].transpose(0, 1).reshape(n, -1, d).float()], 1)
            V = torch.cat([s.V_pre[p, h:h + n].float(), s.V_pages[pages, h:h + n].transpose(0, 1).reshape(n, -1, d).float()], 1)
            x = q[b, :, h * G:(h + n) * G].float().transpose(0, 1).reshape(n, G * T, d)
            score = (x @ K.transpose(1, 2)).view(n, G, T, -1) * (1.0 / math.sqrt(d))
            shown = torch.cat([(states[None, :] < s.prefix_lens[p, h:h + n, None])[:, None, :].expand(n, T, cap),
                               seen[None].expand(n, T, -1)], 2)[:, None]
            score = score.masked_fill_(~shown, float("-inf"))
            top = score.amax(dim=3, keepdim=True)
            weight = torch.exp(score - top)
            total = weight.sum(dim=3, keepdim=True)
            mean = (weight.view(n, G * T, -1) @ V).view(n, G, T, d) / total
            mean = mean.reshape(n * G, T, d).transpose(0, 1).to(dt)
            keep = valid[:, None]
            rows = s.out[b, :, h * G:(h + n) * G]
            rows.copy_(torch.where(keep[..., None], mean, rows))
            if s.lse is not None:
                value = (top + torch.log(total)).reshape(n * G, T).transpose(0, 1)
                rows = s.lse[b, :, h * G:(h + n) * G]
                rows.copy_(torch.where(keep, value, rows))


def exact(case, seed):
    """The outputs in 64 bits, head by head over exactly the keys that a query sees."""
    s = prepare(case, seed)
    new, past = s.new_lens.tolist(), s.past_lens.tolist()
    table = s.table.tolist()
    B, H, G, page = case["B"], s.H, s.G, s.page
    outputs = []
    q = s.q.double()
    K_pages, V_pages = s.K_pages.double(), s.V_pages.double()
    if s.kind != "attn":
        half = s.rot // 2
        freq = s.inv_freq.double()
        q_out = s.q_out.double()
        for b in range(B):
            n = new[b]
            at = past[b] + torch.arange(n, device="cuda")
            phase = (s.pos_base[b].double() + at.double())[:, None, None] * freq
            turn = torch.polar(torch.ones_like(phase), phase)                            # (n, 1, half) unit complex numbers
            where = torch.tensor([table[b][j // page] for j in range(past[b], past[b] + n)], device="cuda")
            for name, x in (("q", q[b, :n]), ("k", s.k[b, :n].double())):
                first = torch.arange(half, device="cuda") * (2 if s.interleaved else 1)
                second = first + (1 if s.interleaved else half)
                z = torch.complex(x[..., first], x[..., second]) * turn
                y = x.clone()
                y[..., first], y[..., second] = z.real, z.imag
                if name == "q":
                    q_out[b, :n] = y
                else:
                    K_pages[where, :, at % page] = y
            V_pages[where, :, at % page] = s.v[b, :n].double()
        outputs += [q_out, K_pages, V_pages, s.past_lens + s.new_lens]
        # what the attention reads was rounded to the cache type when it was stored
        q, K_pages = q_out.to(s.q.dtype).double(), K_pages.to(s.q.dtype).double()
    if s.kind == "append":
        return outputs
    out = s.out.double()
    lse = torch.zeros(out.shape[:3], dtype=torch.float64, device="cuda")
    lens = s.prefix_lens.tolist()
    for b in range(B):
        p, n, before = s.row_prefix[b], new[b], past[b]
        total = before + n
        pages = torch.tensor(table[b][:-(-total // page)], device="cuda", dtype=torch.long)
        future = torch.ones((n, total), dtype=torch.bool, device="cuda").triu(before + 1)
        for h in range(H):
            L = lens[p][h]
            own_k = K_pages[pages, h].reshape(-1, HEAD_DIM)[:total]
            own_v = V_pages[pages, h].reshape(-1, HEAD_DIM)[:total]
            for g in range(G):
                x = q[b, :n, h * G + g] / math.sqrt(HEAD_DIM)
                score = torch.cat([x @ s.K_pre[p, h, :L].double().T,
                                   (x @ own_k.T).masked_fill(future, -math.inf)], 1)
                log_sum = torch.logsumexp(score, dim=1)
                weight = torch.exp(score - log_sum[:, None])
                out[b, :n, h * G + g] = weight[:, :L] @ s.V_pre[p, h, :L].double() + weight[:, L:] @ own_v
                lse[b, :n, h * G + g] = log_sum
    outputs += [out] if s.kind == "step" else [out, lse]
    return outputs


def work(case):
    H, G, esz = case["H"], case["G"], 4 if case["dtype"] == "f32" else 2
    row = HEAD_DIM * esz
    new, tail = np.array(new_lengths(case), dtype=np.float64), np.array(tail_lengths(case), dtype=np.float64)
    tokens = float(new.sum())
    moved, flops = 0.0, 0.0
    if case["kind"] != "attn":
        moved += 2 * tokens * (G + 2) * H * row               # queries, keys, values read, and written
        flops += tokens * (G + 1) * H * 3 * case["rot"]
    if case["kind"] != "append":
        lens, starts = prefix_lengths(case).astype(np.float64), row_starts(case)
        moved += 2 * (float(lens.sum()) + H * float(tail.sum())) * row       # prefixes once, tails once
        moved += tokens * G * H * (2 * row + (4 if case["kind"] == "attn" else 0))
        for p in range(case["P"]):
            rows = slice(starts[p], starts[p + 1])
            seen_own = float((new[rows] * tail[rows] - new[rows] * (new[rows] - 1) / 2).sum())
            flops += 4 * HEAD_DIM * G * (float(new[rows].sum()) * float(lens[p].sum()) + H * seen_own)
    return {"bytes": moved, "flops": flops}
