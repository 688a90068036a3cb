"""Answering from a compacted cache on the GPU, through the C ABI, against the plain 64-bit forms of answer_ref.py: appending to a paged
cache with the position rotation, attention over shared prefixes and paged tails, and both after a compression pass.

Everything that a call must not look at holds NaN: rows behind a prefix's states, slots behind a row's tokens, pages in no row,
tokens that are padding.  Outputs that a call must leave alone hold a pattern."""
import math
import sys

import numpy as np
import pytest
import torch

from paper_2407_08454_amd import binding as kb
from paper_2407_08454_amd import synth

import answer_ref as ar
import gpu_util as gu

pytestmark = pytest.mark.gpu

MARK = 7.0                                                     # exact in every type


def _say(msg):
    print(msg, file=sys.stderr, flush=True)


def _stored(x, dtype):
    """Rounded to dtype, as float64 and on the device."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(gu.TORCH_DT[dtype])
    return t.double().numpy(), t.cuda()


def _i32(x):
    return None if x is None else torch.as_tensor(np.asarray(x, dtype=np.int32)).cuda()


def _check(got, want, tol, what):
    got = gu.to_host_f64(got)
    same = (got == want) | (np.isnan(got) & np.isnan(want))       # equal, infinities included
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= tol))
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} off, first at {np.argwhere(bad)[0].tolist()}: "
                           f"{got[bad][0]} for {want[bad][0]} +- {np.broadcast_to(tol, got.shape)[bad][0]}")


# ---------------------------------------------------------------------------------------------
# appending
# ---------------------------------------------------------------------------------------------

def _append_case(dtype, B, T, H, G, page, rot, interleaved, new, past, pos, seed, fused=True, spoil=None, in_place=False, queries=True,
                 run=None):
    rng = np.random.default_rng(seed)
    freq = (1.0 / 10000.0 ** (np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)
    kv = [p + n for p, n in zip(past, new)]
    table, n_pages = ar.scattered_pages(rng, B, kv, page)
    if spoil:
        spoil(table, n_pages)
    heads = (G + 2) * H
    x64, x = _stored(rng.standard_normal((B, T, heads, 128)), dtype)
    for b in range(B):
        x64[b, new[b]:] = np.nan
        x[b, new[b]:] = float("nan")
    q64, k64, v64 = x64[:, :, :G * H], x64[:, :, G * H:G * H + H], x64[:, :, G * H + H:]
    q, k, v = x[:, :, :G * H], x[:, :, G * H:G * H + H], x[:, :, G * H + H:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    tdt = gu.TORCH_DT[dtype]
    Kp, Vp = (torch.full((n_pages, H, page, 128), MARK, dtype=tdt, device="cuda") for _ in range(2))
    q_out = (q if in_place else torch.full((B, T, G * H, 128), MARK, dtype=tdt, device="cuda")) if queries else None
    before = q64.copy() if in_place else np.full(q64.shape, MARK)
    kv_lens = torch.full((B,), -5, dtype=torch.int32, device="cuda")
    pages = kb.make_pages(Kp, Vp, torch.from_numpy(table).cuda())
    shape = kb.make_token_shape(pages, T, G, _i32(new))
    rotation = kb.make_rotation(torch.from_numpy(freq).cuda() if rot else None, interleaved)
    call = lambda: kb.kvm_paged_append(shape, pages, rotation, q if queries else None, k, v, _i32(past), _i32(pos), q_out, kv_lens)
    (run or (lambda f: f()))(call)
    torch.cuda.synchronize()
    want = ar.append(q64 if queries else None, k64, v64, new, past, pos or [0] * B, freq, interleaved, np.full(Kp.shape, MARK),
                     np.full(Vp.shape, MARK), table, before)
    half = ar.EPS[dtype] / 2
    # the angle's fraction of a turn is rounded to fp32 and the two functions are off by a few of their last places: sine and cosine
    # within 2^-21, products and difference another 2^-23 of the pair's length; one rounding to dtype
    for got, ref, size, name in ((q_out, want[0], want[4], "q_out"), (Kp, want[1], want[5], "keys"), (Vp, want[2], 0.0, "values")):
        if got is not None:
            tol = (2.0 ** -20 * size) * (1 + 2 * half) + np.where(np.asarray(size) > 0, half * np.abs(ref) + ar.TINY[dtype] / 2, 0.0)
            _check(got, ref, tol, name)
    assert kv_lens.tolist() == want[3].tolist()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [128, 64, 16, 0])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_append_rotations(dtype, rot, interleaved):
    _say(f"append {dtype} rot={rot} interleaved={interleaved}")
    _append_case(dtype, 3, 4, 2, 2, 4, rot, interleaved, [4, 1, 3], [0, 6, 3], [0, 5000, 123456], 1)


@pytest.mark.parametrize("dtype,B,T,H,G,page,new,past,pos", [
    ("f16", 1, 1, 1, 1, 16, [1], [0], None),                                     # one token, one head
    ("bf16", 1, 1, 32, 1, 16, [1], [31], [4096]),                                # the last slot of a page
    ("f16", 70, 1, 8, 4, 64, [1] * 70, list(range(70)), list(range(70))),        # a decoding batch
    ("f32", 5, 1, 5, 7, 1, [1, 0, 1, 0, 1], [3, 2, 1, 0, 9], [9, 8, 7, 6, 5]),   # pages of one token, rows without a new one
    ("bf16", 2, 133, 3, 1, 32, [133, 40], [17, 100], [2 ** 22, 2 ** 30]),        # chunks that start inside a page, far positions
    ("f16", 4, 9, 1, 33, 8, [9, 0, 0, 9], [0, 0, 16, 15], [0, 1, 2, -40]),       # an odd number of heads, rows of nothing, negative positions
    ("f32", 2, 600, 4, 2, 128, [600, 599], [0, 1], [1000000, 2000000000]),
    ("f16", 300, 2, 2, 1, 16, [i % 3 for i in range(300)], [0] * 300, [1] * 300),   # more rows than a workgroup adds up
])
@pytest.mark.parametrize("fused", [True, False])
def test_append_sizes(dtype, B, T, H, G, page, new, past, pos, fused):
    _say(f"append {dtype} B={B} T={T} H={H} G={G} page={page} fused={fused}")
    _append_case(dtype, B, T, H, G, page, 128, False, new, past, pos, 2, fused)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pos", [0, 1000000])
def test_append_angles_are_rounded_once(pos, interleaved):
    """fp32: pairs (1, 0) become cosine and sine, each off by half a step at one, 2^-25, and by what the angle x f loses in 64 bits (two
    roundings in the kernel, one and the functions' own in numpy)."""
    T, H = 1500, 1
    freq = (1.0 / 10000.0 ** (np.arange(0, 128, 2) / 128)).astype(np.float32)
    x = torch.zeros((1, T, 3, 128), device="cuda")
    x[..., 0::2] = 1.0
    if not interleaved:
        x[..., :64], x[..., 64:] = 1.0, 0.0
    pool = [torch.zeros((-(-T // 64), H, 64, 128), device="cuda") for _ in range(2)]
    pages = kb.make_pages(*pool, torch.arange(len(pool[0]), dtype=torch.int32, device="cuda")[None])
    q_out, kv = torch.empty((1, T, 1, 128), device="cuda"), _i32([0])
    kb.kvm_paged_append(kb.make_token_shape(pages, T, 1), pages, kb.make_rotation(torch.from_numpy(freq).cuda(), interleaved), x[:, :, :1],
                        x[:, :, 1:2], x[:, :, 2:], _i32([0]), _i32([pos]), q_out, kv)
    angle = (pos + np.arange(T, dtype=np.float64))[:, None] * freq.astype(np.float64)
    want = np.stack([np.cos(angle), np.sin(angle)], 2 if interleaved else 1).reshape(T, 128)
    tol = np.stack([2.0 ** -25 + 2.0 ** -50 * (1 + np.abs(angle))] * 2, 2 if interleaved else 1).reshape(T, 128)
    _check(q_out[0, :, 0], want, tol, "queries")
    _check(pool[0][:, 0].reshape(-1, 128)[:T], want, tol, "keys")


@pytest.mark.parametrize("dtype,B,T", [("f16", 3, 7000), ("f32", 2, 5500)])
def test_append_of_more_than_the_last_level_cache(dtype, B, T):
    """Large steps take the streaming kernel: rows of both ends against the plain form, and every value row against its source."""
    H, G, page, tdt = 16, 2, 64, gu.TORCH_DT[dtype]
    n_pages = B * (T // page + 2)
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((B, T, (G + 2) * H, 128), generator=gen, device="cuda").to(tdt)
    assert 2 * x.nbytes >= 256 << 20
    Kp, Vp = (torch.full((n_pages, H, page, 128), MARK, dtype=tdt, device="cuda") for _ in range(2))
    table = torch.randperm(n_pages, device="cuda").to(torch.int32).view(B, -1)
    new, past, pos = [T, T - 77, 5][:B], [3, 0, 60][:B], [1000, 0, 7][:B]
    pages = kb.make_pages(Kp, Vp, table)
    freq = (1.0 / 10000.0 ** (np.arange(0, 128, 2) / 128)).astype(np.float32)
    q_out, kv = torch.full((B, T, G * H, 128), MARK, dtype=tdt, device="cuda"), _i32([0] * B)
    HG = G * H
    kb.kvm_paged_append(kb.make_token_shape(pages, T, G, _i32(new)), pages, kb.make_rotation(torch.from_numpy(freq).cuda(), True), x[:, :, :HG],
                        x[:, :, HG:HG + H], x[:, :, HG + H:], _i32(past), _i32(pos), q_out, kv)
    assert kv.tolist() == [p + n for p, n in zip(past, new)]
    assert (q_out[1, new[1]:] == MARK).all()
    for b in range(B):
        slot = past[b] + torch.arange(new[b], device="cuda")
        where = table[b].long()[slot // page]
        assert torch.equal(Vp[where, :, slot % page], x[b, :new[b], HG + H:])
        for t in {0, 1, new[b] // 2, new[b] - 1}:
            turned = ar.rotate(gu.to_host_f64(x[b, t, :HG + H]), np.full(HG + H, pos[b] + past[b] + t), freq, True)
            got = torch.cat([q_out[b, t], Kp[where[t], :, slot[t] % page]])
            length = np.repeat(np.hypot(*(gu.to_host_f64(x[b, t, :HG + H])[:, i::2] for i in (0, 1))), 2, axis=1)
            half = ar.EPS[dtype] / 2
            _check(got, turned, 2.0 ** -20 * length * (1 + 2 * half) + half * np.abs(turned) + ar.TINY[dtype], f"row {b} token {t}")


def test_append_without_queries_and_in_place():
    _append_case("bf16", 3, 5, 2, 3, 16, 64, True, [5, 2, 0], [1, 14, 3], [7, 8, 9], 3, queries=False)
    _append_case("f16", 3, 5, 2, 3, 16, 64, False, [5, 2, 0], [1, 14, 3], [7, 8, 9], 4, fused=False, in_place=True)


def test_append_leaves_out_pages_that_a_row_does_not_have():
    """Entries outside the pool, and slots behind the table: nothing is stored there, the rest of the call is as ever."""
    def spoil(table, n_pages):
        table[0, 1], table[1, 0], table[2, 1] = -1, n_pages, 2 ** 31 - 1
    _append_case("f16", 3, 20, 2, 1, 8, 128, False, [20, 5, 20], [0, 2, 3], None, 5, spoil=spoil)
    _say("append behind the table")
    page, tdt = 4, torch.float16
    for past, new, kv in ((7, 3, 8), (8, 2, 8), (100, 1, 8), (-3, 2, 2)):
        pool = [torch.full((2, 1, page, 128), MARK, dtype=tdt, device="cuda") for _ in range(2)]
        pages = kb.make_pages(*pool, _i32([[0, 1]]))
        x = torch.ones((1, new, 3, 128), dtype=tdt, device="cuda")
        q_out, kv_lens = torch.zeros((1, new, 1, 128), dtype=tdt, device="cuda"), _i32([0])
        kb.kvm_paged_append(kb.make_token_shape(pages, new, 1), pages, kb.make_rotation(), x[:, :, :1], x[:, :, 1:2], x[:, :, 2:], _i32([past]),
                            None, q_out, kv_lens)
        assert kv_lens.item() == kv and (q_out == 1).all()
        for t in pool:
            slots = t.view(8, 128)
            first = max(past, 0)
            assert (slots[min(first, 8):min(first + new, 8)] == 1).all() and int((slots == 1).sum()) == 128 * (kv - min(first, 8))


def test_append_beyond_32_bits():
    """A pool of more than 2^32 elements: the last page."""
    H, page = 32, 64
    n_pages = 2 ** 32 // (H * page * 128) + 3
    Kp, Vp = (torch.empty((n_pages, H, page, 128), dtype=torch.float16, device="cuda") for _ in range(2))
    pages = kb.make_pages(Kp, Vp, _i32([[n_pages - 1], [0]]))
    x = torch.randn((2, 1, 3 * H, 128), device="cuda").half()
    q_out, kv = torch.empty((2, 1, H, 128), dtype=torch.float16, device="cuda"), _i32([0, 0])
    kb.kvm_paged_append(kb.make_token_shape(pages, 1, 1), pages, kb.make_rotation(), x[:, :, :H], x[:, :, H:2 * H], x[:, :, 2 * H:],
                        _i32([63, 1]), None, q_out, kv)
    for row, (p, at) in enumerate(((n_pages - 1, 63), (0, 1))):
        assert torch.equal(Kp[p, :, at], x[row, 0, H:2 * H]) and torch.equal(Vp[p, :, at], x[row, 0, 2 * H:])
    assert torch.equal(q_out, x[:, :, :H]) and kv.tolist() == [64, 2]


# ---------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------

class Attn:
    """Inputs of one call, on the host in 64 bits and on the device."""

    def __init__(self, dtype, B, T, H, G, seed, P=0, cap=0, lens=None, row_start=None, kv=None, page=16, new=None, q_scale=1.0, strided=False,
                 spoil=None):
        rng = np.random.default_rng(seed)
        self.dtype, self.B, self.T, self.H, self.G, self.new = dtype, B, T, H, G, new
        x64, x = _stored(rng.standard_normal((B, T, H * G + (2 if strided else 0), 128)) * q_scale, dtype)
        for b in range(B):
            if new is not None:
                x[b, new[b]:] = float("nan")
        self.q64, self.q = x64[:, :, :H * G], x[:, :, :H * G]
        self.prefix = self.pages = self.prefix64 = self.pages64 = None
        if P or cap:
            K, V = rng.standard_normal((P, H, cap, 128)), rng.standard_normal((P, H, cap, 128))
            if lens is not None:
                lens = np.broadcast_to(np.asarray(lens, np.int32), (P, H)).copy()
                for p in range(P):
                    for h in range(H):
                        K[p, h, max(lens[p, h], 0):], V[p, h, max(lens[p, h], 0):] = np.nan, np.nan
            (K64, Kd), (V64, Vd) = _stored(K, dtype), _stored(V, dtype)
            self.prefix64 = dict(K=K64, V=V64, lens=lens, row_start=row_start)
            self.prefix = kb.make_prefix(Kd, Vd, _i32(lens), _i32(row_start))
        if kv is not None:
            table, n_pages = ar.scattered_pages(rng, B, [max(n, 0) for n in kv], page)
            K, V = np.full((n_pages, H, page, 128), np.nan), np.full((n_pages, H, page, 128), np.nan)
            for b in range(B):
                for j in range(kv[b]):
                    K[table[b, j // page], :, j % page] = rng.standard_normal((H, 128))
                    V[table[b, j // page], :, j % page] = rng.standard_normal((H, 128))
            if spoil:
                spoil(table, n_pages, K, V)
            (K64, Kd), (V64, Vd) = _stored(K, dtype), _stored(V, dtype)
            self.pages64 = dict(K=K64, V=V64, table=table, kv_lens=kv)
            self.pages = kb.make_pages(Kd, Vd, torch.from_numpy(table).cuda())
        self.kv_lens = _i32(kv)
        if self.pages is not None:
            self.shape = kb.make_token_shape(self.pages, T, G, _i32(new))
        else:
            self.shape = kb.make_token_shape(self.prefix, T, G, _i32(new), B=B)
        self.out = torch.empty((B, T, H * G, 128), dtype=gu.TORCH_DT[dtype], device="cuda")
        self.lse = torch.empty((B, T, H * G), dtype=torch.float32, device="cuda")
        self.ws = torch.empty(kb.kvm_prefix_attn_workspace_bytes(self.shape, self.prefix, self.pages), dtype=torch.uint8, device="cuda")

    def call(self, lse=True):
        kb.kvm_prefix_attn(self.shape, self.prefix, self.pages, self.q, self.kv_lens, self.out, self.lse if lse else None, self.ws)

    def run(self):
        self.out.fill_(MARK)
        self.lse.fill_(MARK)
        self.ws.fill_(255)                                     # NaN, should anything be read that was not written
        self.call()
        torch.cuda.synchronize()
        return self

    def check(self):
        out, lse, bounds = ar.attention(self.q64, self.G, self.new, self.prefix64, self.pages64)
        o_tol, l_tol = ar.tolerance(self.dtype, out, lse, bounds)
        there = ~np.isnan(lse)
        out[~there], lse[~there], o_tol[~there], l_tol[~there] = MARK, MARK, 0.0, 0.0
        _check(self.lse, lse, l_tol, "lse")
        _check(self.out, out, o_tol, "out")
        return self


CASES = {
    # one row, one token: one key, and a few
    "one_key": dict(B=1, T=1, H=1, G=1, kv=[1]),
    "one_state": dict(B=1, T=1, H=2, G=1, P=1, cap=1),
    "tiny": dict(B=2, T=1, H=2, G=2, P=1, cap=5, kv=[1, 2], page=1),
    # a single row over a cache of ordinary size
    "single_row": dict(B=1, T=1, H=4, G=1, P=1, cap=2048, lens=[[2048, 1999, 1280, 33]], kv=[100]),
    # rows that share a prefix: counts around a tile of 32 query rows, odd states
    "rows_31": dict(B=31, T=1, H=2, G=1, P=1, cap=77, kv=list(range(1, 32)), page=4),
    "rows_33": dict(B=33, T=1, H=2, G=1, P=1, cap=129, lens=[[129, 64]], kv=[5] * 33),
    "rows_130_g4": dict(B=130, T=1, H=1, G=4, P=1, cap=400, kv=[(7 * i) % 50 + 1 for i in range(130)]),
    "many_rows_ragged": dict(B=150, T=2, H=2, G=1, P=2, cap=300, lens=[[300, 0], [129, 64]], row_start=[3, 100, 149], kv=[2 + (5 * i) % 70 for i in range(150)]),
    "many_rows_prefix_alone": dict(B=140, T=1, H=1, G=2, P=2, cap=190, lens=[[190], [65]]),
    "g33": dict(B=3, T=1, H=1, G=33, P=1, cap=100, kv=[64, 65, 1]),
    # prompts with different numbers of rows, one without rows, rows of no prompt
    "ragged_prompts": dict(B=41, T=1, H=2, G=2, P=5, cap=200, lens=[[200, 3], [0, 150], [7, 7], [64, 65], [1, 0]], row_start=[1, 4, 4, 37, 39, 40],
                           kv=[(11 * i) % 90 for i in range(41)]),
    "many_prompts": dict(B=90, T=1, H=1, G=2, P=90, cap=33, lens=[[i % 34] for i in range(90)], kv=[i % 5 for i in range(90)], page=2),
    # nothing to see for a head or a row
    "empty": dict(B=4, T=2, H=2, G=2, P=2, cap=40, lens=[[0, 40], [0, 0]], kv=[0, 3, 0, 1]),
    "all_empty": dict(B=2, T=1, H=1, G=1, P=1, cap=8, lens=[[0]], kv=[0, 0]),
    "negative_lens": dict(B=2, T=1, H=1, G=1, P=1, cap=8, lens=[[-4]], kv=[-1, 3]),
    # several tokens a row: drafts, chunks, padding, rows without tokens, tails shorter than the new tokens
    "drafts": dict(B=10, T=3, H=2, G=2, P=2, cap=143, lens=[[143, 20], [90, 91]], kv=[3 * i + 3 for i in range(10)], new=[3, 2, 1, 0, 3, 3, 3, 2, 1, 3]),
    "short_kv": dict(B=2, T=4, H=1, G=1, P=1, cap=9, kv=[2, 0]),
    "chunk_70": dict(B=3, T=70, H=2, G=3, P=1, cap=200, lens=[[200, 61]], kv=[300, 70, 71], new=[70, 70, 9]),
    "chunk_333": dict(B=2, T=333, H=1, G=2, P=2, cap=77, kv=[333, 1001], new=[300, 333], page=64),
    "chunk_alone": dict(B=1, T=257, H=2, G=1, kv=[257], page=128),
    "chunk_b8": dict(B=8, T=40, H=1, G=1, P=2, cap=500, kv=[40 + 13 * i for i in range(8)], new=[40 - i for i in range(8)], page=32),
    # long axes
    "long_prefix": dict(B=2, T=1, H=1, G=1, P=1, cap=20011, kv=[1, 40]),
    "long_tail": dict(B=2, T=1, H=1, G=2, P=1, cap=10, kv=[9001, 317], page=128),
    "long_both_t2": dict(B=2, T=2, H=1, G=1, P=2, cap=5000, lens=[[5000], [4097]], kv=[6000, 2], page=64),
    # pages of one token (a tile takes as many entries of the table as are held at once), pages longer than most rows
    "pages_of_one": dict(B=3, T=1, H=2, G=1, P=1, cap=10, kv=[500, 64, 65], page=1),
    "pages_of_one_chunk": dict(B=2, T=140, H=1, G=1, P=1, cap=70, kv=[300, 141], page=1),
    "pages_of_two_chunk": dict(B=1, T=70, H=1, G=2, kv=[401], page=2),
    "long_pages": dict(B=2, T=1, H=1, G=2, kv=[1500, 3], page=1024),
    "long_pages_chunk": dict(B=2, T=150, H=1, G=1, P=1, cap=64, kv=[1100, 150], page=1024),
    # a prefix alone (another length than the queries'), pages alone
    "prefix_alone": dict(B=3, T=50, H=2, G=2, P=3, cap=333, lens=[[333, 100], [1, 0], [32, 33]], new=[50, 20, 3]),
    "pages_alone": dict(B=5, T=1, H=3, G=2, kv=[1, 16, 17, 0, 500]),
    "strided": dict(B=3, T=4, H=2, G=2, P=1, cap=60, kv=[4, 5, 60], strided=True),
    # scores far apart: weights of a few keys only
    "sharp": dict(B=4, T=2, H=1, G=2, P=1, cap=300, kv=[100, 2, 40, 3], q_scale=30.0),
    "sharp_chunk": dict(B=1, T=100, H=1, G=1, P=1, cap=300, kv=[170], q_scale=30.0),
}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", list(CASES))
def test_attention(name, dtype):
    _say(f"attention {name} {dtype}")
    Attn(dtype, seed=11, **CASES[name]).run().check()


@pytest.mark.parametrize("name,kernels", [
    ("single_row", {"prefix_attn_split_kernel", "prefix_attn_join_kernel"}),
    ("rows_33", {"prefix_attn_split_kernel", "prefix_attn_join_kernel"}),
    ("rows_130_g4", {"prefix_attn_wide_kernel", "prefix_attn_join_kernel"}),           # 520 queries of a prompt
    ("many_rows_ragged", {"prefix_attn_wide_kernel", "prefix_attn_join_kernel"}),
    ("chunk_333", {"prefix_attn_wide_kernel", "prefix_attn_join_kernel"}),             # few tiles: their keys in parts
    ("all_empty", {"prefix_attn_split_kernel", "prefix_attn_join_kernel"}),
])
def test_which_kernels_run(name, kernels):
    a = Attn("bf16", seed=3, **CASES[name])
    assert gu.kernels_of(a.call) == kernels


def test_many_tokens_go_straight_to_the_output():
    """Enough query tiles for the chip: prefix and tail in one pass, nothing to join."""
    a = Attn("f16", B=9, T=100, H=8, G=10, seed=8, P=3, cap=70, lens=[[70] * 8, [1] * 8, [0] * 8], kv=[100 + i for i in range(9)], new=[100 - 11 * i for i in range(9)])
    assert gu.kernels_of(a.call) == {"prefix_attn_wide_kernel"}
    rows = [0, 4, 8]                                           # (the plain form of all of them takes long)
    a.run()
    for b in rows:
        p = b // 3
        out, lse, bounds = ar.attention(a.q64[b:b + 1], a.G, a.new[b:b + 1], dict(K=a.prefix64["K"][p:p + 1], V=a.prefix64["V"][p:p + 1],
                                        lens=a.prefix64["lens"][p:p + 1], row_start=None), dict(a.pages64, table=a.pages64["table"][b:b + 1], kv_lens=a.pages64["kv_lens"][b:b + 1]))
        o_tol, l_tol = ar.tolerance("f16", out, lse, bounds)
        there = ~np.isnan(lse)
        out[~there], lse[~there], o_tol[~there], l_tol[~there] = MARK, MARK, 0.0, 0.0
        _check(a.lse[b:b + 1], lse, l_tol, f"lse of row {b}")
        _check(a.out[b:b + 1], out, o_tol, f"out of row {b}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T", [1, 40])
def test_attention_does_not_see_pages_that_a_row_does_not_have(dtype, T):
    def spoil(table, n_pages, K, V):
        table[0, 1], table[1, 0], table[1, 2], table[2, 3] = -1, n_pages, 2 ** 31 - 1, -2 ** 31
    _say(f"missing pages {dtype} T={T}")
    Attn(dtype, 3, T, 2, 2, 5, P=1, cap=50, kv=[45, 70, 64], page=16, spoil=spoil).run().check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,G", [(3, 2), (40, 1), (200, 2)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_later_token_has_no_influence(dtype, T, G, value):
    """Keys and values of later tokens of the same step are in the pages already: infinities and NaN there reach no earlier query."""
    _say(f"later token {dtype} T={T} G={G} {value}")
    last = T // 2 + 1                                          # the first token that is spoilt
    kv = [T + 9, T]

    def spoil(table, n_pages, K, V):
        for b in range(2):
            for j in range(kv[b] - T + last, kv[b]):
                K[table[b, j // 16], :, j % 16, j % 128] = value
                V[table[b, j // 16], :, j % 16, (3 * j) % 128] = value

    a = Attn(dtype, 2, T, 2, G, 6, P=1, cap=45, kv=kv, spoil=spoil).run()
    out, lse, bounds = ar.attention(a.q64[:, :last], G, None, a.prefix64, dict(a.pages64, kv_lens=[n - T + last for n in kv]))
    o_tol, l_tol = ar.tolerance(dtype, out, lse, bounds)
    _check(a.out[:, :last], out, o_tol, "out")
    _check(a.lse[:, :last], lse, l_tol, "lse")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,rows", [(1, 3), (1, 200), (5, 3), (150, 2)])
def test_an_infinite_value_that_is_seen_stays_infinite(dtype, T, rows):
    """One infinity among a prefix's values and one among a tail's: in their dimensions of the queries that see them, nowhere else."""
    _say(f"infinite value {dtype} T={T} rows={rows}")

    def spoil(table, n_pages, K, V):
        V[table[1, 0], 1, 2, 5] = -np.inf                      # token 2 of row 1, KV head 1

    a = Attn(dtype, rows, T, 2, 2, 15, P=1, cap=90, lens=[[90, 70]], kv=[T + 40] * rows, spoil=spoil)
    a.prefix64["V"][0, 0, 33, 7] = np.inf
    a.prefix._refs[1][0, 0, 33, 7] = float("inf")
    a.run()
    few = min(rows, 3)
    out, lse, bounds = ar.attention(a.q64[:few], 2, None, a.prefix64, dict(a.pages64, table=a.pages64["table"][:few], kv_lens=a.pages64["kv_lens"][:few]))
    o_tol, l_tol = ar.tolerance(dtype, out, lse, tuple(np.nan_to_num(x, posinf=0.0) for x in bounds))
    assert np.isposinf(out[:, :, :2, 7]).all() and np.isneginf(out[1, :, 2:, 5]).all() and np.isinf(out).sum() == few * T * 2 + T * 2
    _check(a.out[:few], out, o_tol, "out")
    _check(a.lse[:few], lse, l_tol, "lse")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,rows,H", [(1, 3, 2), (1, 200, 2), (150, 2, 2), (130, 65, 4)])
def test_an_infinite_value_under_a_small_weight_stays_infinite(dtype, T, rows, H):
    """The same where the weight is e^-30 of the greatest, which 16 bits do not hold: one among a prefix's values, one in the tail of a row,
    long before its new tokens.  The last shape goes straight to the output."""
    _say(f"infinite value, small weight {dtype} T={T} rows={rows}")
    a = Attn(dtype, rows, T, H, 1, 18, P=1, cap=150, kv=[T + 190] * rows)
    put = lambda x64, x, at, value: (x64.__setitem__(at, value), x.__setitem__(at, value))
    every = np.s_[:]
    put(a.q64, a.q, every, 0.0)
    put(a.q64, a.q, np.s_[..., 0], 14.25)
    (pre_k, pre_v, _, _), (own_k, own_v, _) = a.prefix._refs, a.pages._refs
    put(a.prefix64["K"], pre_k, every, 0.0)
    put(a.pages64["K"], own_k, every, 0.0)
    put(a.prefix64["K"], pre_k, np.s_[:, :, 0, 0], 24.0)       # 14.25 * 24 / sqrt(128) = 30.2
    put(a.prefix64["V"], pre_v, np.s_[0, 0, 133, 7], np.inf)
    put(a.pages64["V"], own_v, np.s_[a.pages64["table"][1, 4], 1, 2, 5], -np.inf)      # token 66 of row 1, KV head 1
    a.run()
    assert (a.out == MARK).sum() == 0
    few = 2 if T > 1 else 3
    out, lse, bounds = ar.attention(a.q64[:few], 1, None, a.prefix64, dict(a.pages64, table=a.pages64["table"][:few], kv_lens=a.pages64["kv_lens"][:few]))
    o_tol, l_tol = ar.tolerance(dtype, out, lse, tuple(np.nan_to_num(x, posinf=0.0) for x in bounds))
    assert np.isposinf(out[:, :, 0, 7]).all() and np.isneginf(out[1, :, 1, 5]).all() and np.isinf(out).sum() == few * T + T
    _check(a.out[:few], out, o_tol, "out")
    _check(a.lse[:few], lse, l_tol, "lse")
    assert torch.isinf(a.out).sum().item() == rows * T + T and not torch.isnan(a.out).any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,rows,H", [(1, 3, 2), (1, 200, 2), (150, 2, 2), (130, 65, 4)])
@pytest.mark.parametrize("page", [2, 64])
def test_a_nan_that_is_seen_stays_in_its_dimension(dtype, T, rows, H, page):
    """Also what two infinities of different signs make; beside them an infinity that is seen, and a NaN that only the last token sees."""
    _say(f"seen NaN {dtype} T={T} rows={rows} page={page}")
    a = Attn(dtype, rows, T, H, 1, 22, P=1, cap=150, kv=[T + 190] * rows, page=page)
    put = lambda x64, x, at, value: (x64.__setitem__(at, value), x.__setitem__(at, value))
    (_, pre_v, _, _), (_, own_v, _) = a.prefix._refs, a.pages._refs
    own = lambda b, j, d: np.s_[a.pages64["table"][b, j // page], 1, j % page, d]
    put(a.prefix64["V"], pre_v, np.s_[0, 0, 133, 7], np.nan)
    put(a.prefix64["V"], pre_v, np.s_[0, 0, 2, 8], np.inf)
    put(a.prefix64["V"], pre_v, np.s_[0, 1, 3, 127], -np.inf)
    put(a.pages64["V"], own_v, own(0, 71, 127), np.inf)        # meets the last one, in row 0 alone
    put(a.pages64["V"], own_v, own(1, 5, 0), -np.inf)
    put(a.pages64["V"], own_v, own(1, T + 189, 1), np.nan)     # the last token's own
    a.run()
    assert (a.out == MARK).sum() == 0
    few = 2 if T > 1 else 3
    with np.errstate(invalid="ignore"):                        # inf - inf is meant
        want, lse, bounds = ar.attention(a.q64[:few], 1, None, a.prefix64, dict(a.pages64, table=a.pages64["table"][:few], kv_lens=a.pages64["kv_lens"][:few]))
    o_tol, l_tol = ar.tolerance(dtype, want, lse, tuple(np.nan_to_num(x, nan=0.0, posinf=0.0) for x in bounds))
    nans = np.zeros(want.shape, bool)
    nans[:, :, 0, 7], nans[0, :, 1, 127], nans[1, T - 1, 1, 1] = True, True, True
    assert (np.isnan(want) == nans).all() and np.isinf(want).sum() == few * T + (few - 1) * T + T
    o_tol[~np.isfinite(want)] = 0.0
    _check(a.out[:few], want, o_tol, "out")
    _check(a.lse[:few], lse, l_tol, "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,rows,H", [(1, 3, 1), (1, 200, 1), (150, 2, 1), (130, 65, 4)])
def test_great_values_under_a_reference_that_lags(dtype, T, rows, H):
    """A later state with a score five above the ones before it has a weight of 2^7 against their reference: with a value of 2^125 the sum is beyond
    fp32, though the output is not."""
    _say(f"great values {dtype} T={T} rows={rows}")
    a = Attn(dtype, rows, T, H, 1, 23, P=1, cap=150)
    a.prefix64["K"][...] = 0.0
    a.prefix64["K"][:, :, 130, 0] = 4.0                        # 14.25 * 4 / sqrt(128) = 5.04
    a.prefix64["V"][:, :, 130] = 2.0 ** 125 * (1 - 2 * (np.arange(128) % 2))
    a.q64[...] = 0.0
    a.q64[..., 0] = 14.25
    for x64, x in ((a.prefix64["K"], a.prefix._refs[0]), (a.prefix64["V"], a.prefix._refs[1]), (a.q64, a.q)):
        x.copy_(torch.from_numpy(x64))
    a.run()
    few = min(rows, 2)
    out, lse, bounds = ar.attention(a.q64[:few], 1, None, a.prefix64, None)
    o_tol, l_tol = ar.tolerance(dtype, out, lse, bounds)
    _check(a.out[:few], out, o_tol, "out")
    _check(a.lse[:few], lse, l_tol, "lse")
    assert torch.isfinite(a.out).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,rows", [(1, 2), (1, 200), (150, 2)])
def test_many_small_weights_beside_a_great_one(dtype, T, rows):
    """A first state with nearly all of the weight and a value of zero, as models have them: the output is what thousands of weights of
    e^-18 leave.  In fp16 a weight is off by 2^-25 at most where the greatest is 2^10 or more, so by 2^-35 of the greatest."""
    _say(f"small weights {dtype} T={T} rows={rows}")
    n = 4000
    a = Attn(dtype, rows, T, 1, 1, 16, P=1, cap=n)
    a.prefix64["K"][...] = 0.0
    a.prefix64["K"][0, 0, 0, 0] = 14.25                       # 14.25^2 / sqrt(128) = 17.95
    a.prefix64["V"][...] = 64.0 + np.arange(128) / 2
    a.prefix64["V"][0, 0, 0] = 0.0
    a.q64[...] = 0.0
    a.q64[..., 0] = 14.25
    for x64, x in ((a.prefix64["K"], a.prefix._refs[0]), (a.prefix64["V"], a.prefix._refs[1]), (a.q64, a.q)):
        x.copy_(torch.from_numpy(x64))                        # (exact in every type)
    a.run()
    few = min(rows, 2)
    out, lse, (spread, worst, small) = ar.attention(a.q64[:few], 1, None, a.prefix64, None)
    o_tol, l_tol = ar.tolerance(dtype, out, lse, (spread, worst, small * 2.0 ** -10))
    _check(a.out[:few], out, o_tol, "out")
    _check(a.lse[:few], lse, l_tol, "lse")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,rows,H,G", [(1, 3, 2, 2), (5, 4, 2, 1), (1, 130, 1, 2), (150, 2, 2, 1), (130, 65, 4, 1)])
def test_what_the_rounding_of_a_weight_leaves_is_not_lost(dtype, T, rows, H, G):
    """Few queries, many rows of a prompt, many tokens of a row in parts and straight to the output: in every kernel the weights count with twice
    the bits of their type, so that beside the output's own rounding there is a quarter of a step's square of a weight; small scores
    keep what fp32 sums leave below that.  Weights with one rounding would be outside, as the plain form shows."""
    _say(f"two-part weights {dtype} T={T} rows={rows} G={G}")
    a = Attn(dtype, rows, T, H, G, 19, P=1, cap=12, kv=[T + 5] * rows, q_scale=0.25).run()
    few, half = 2, ar.EPS[dtype] / 2
    own = dict(a.pages64, table=a.pages64["table"][:few], kv_lens=a.pages64["kv_lens"][:few])
    out, lse, (spread, worst, small) = ar.attention(a.q64[:few], G, None, a.prefix64, own)
    tol = (half * half + 2 * worst)[..., None] * spread + (ar.TINY[dtype] / 2 * 2.0 ** -10 * small if dtype == "f16" else 0.0)
    tol = tol * (1 + ar.EPS[dtype]) + half * np.abs(out) + ar.TINY[dtype]
    _check(a.out[:few], out, tol, "out")
    # the first token of row 0, head 0, with weights of one rounding
    K, V = (np.concatenate([a.prefix64[x][0, 0], a.pages64[x][a.pages64["table"][0, 0], 0, :6]]) for x in ("K", "V"))
    w = np.exp(K @ a.q64[0, 0, 0] / math.sqrt(128))
    w /= w.max()
    assert np.allclose(w @ V / w.sum(), out[0, 0, 0], rtol=0, atol=1e-12)
    once = _stored(_stored(w, dtype)[0] @ V / w.sum(), dtype)[0]
    assert (np.abs(once - out[0, 0, 0]) > tol[0, 0, 0]).any()


def test_steps_without_tokens_and_batches_without_rows():
    tdt = torch.float16
    pool = [torch.full((3, 2, 4, 128), MARK, dtype=tdt, device="cuda") for _ in range(2)]
    empty = lambda *s: torch.empty(s, dtype=tdt, device="cuda")
    pages = kb.make_pages(*pool, _i32([[0, 1], [2, -1]]))
    shape, kv = kb.make_token_shape(pages, 0, 2), _i32([-1, -1])
    kb.kvm_paged_append(shape, pages, kb.make_rotation(), empty(2, 0, 4, 128), empty(2, 0, 2, 128), empty(2, 0, 2, 128), _i32([5, 3]), None,
                        empty(2, 0, 4, 128), kv)
    assert kv.tolist() == [5, 3] and all((t == MARK).all() for t in pool)
    ws = torch.empty(kb.kvm_prefix_attn_workspace_bytes(shape, None, pages), dtype=torch.uint8, device="cuda")
    kb.kvm_prefix_attn(shape, None, pages, empty(2, 0, 4, 128), kv, empty(2, 0, 4, 128), None, ws)
    none = kb.make_pages(*pool, torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    shape, kv = kb.make_token_shape(none, 3, 2), torch.empty(0, dtype=torch.int32, device="cuda")
    kb.kvm_paged_append(shape, none, kb.make_rotation(), empty(0, 3, 4, 128), empty(0, 3, 2, 128), empty(0, 3, 2, 128), kv, None,
                        empty(0, 3, 4, 128), torch.empty(0, dtype=torch.int32, device="cuda"))
    kb.kvm_prefix_attn(shape, None, none, empty(0, 3, 4, 128), kv, empty(0, 3, 4, 128), None, ws)
    torch.cuda.synchronize()
    # pools and tables without pages: nothing to see
    bare = kb.make_pages(empty(0, 2, 4, 128), empty(0, 2, 4, 128), torch.empty((2, 0), dtype=torch.int32, device="cuda"))
    shape, out = kb.make_token_shape(bare, 1, 2), torch.full((2, 1, 4, 128), MARK, dtype=tdt, device="cuda")
    ws = torch.empty(kb.kvm_prefix_attn_workspace_bytes(shape, None, bare), dtype=torch.uint8, device="cuda")
    kb.kvm_prefix_attn(shape, None, bare, torch.ones_like(out), _i32([9, 9]), out, None, ws)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,G", [(1, 1), (3, 2), (200, 1)])
def test_a_batch_without_rows_with_the_workspace_of_its_own_size(dtype, T, G):
    """A running batch whose last row has ended: sized, and called, as any other."""
    _say(f"no rows {dtype} T={T} G={G}")
    a = Attn(dtype, 0, T, 2, G, 17, P=1, cap=50, lens=[[50, 7]], row_start=[0, 0], kv=[])
    assert a.ws.numel() == 256
    a.run()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_with_equal_scores_is_the_mean(dtype):
    """Queries of zero: the plain mean of the values, whatever the number of keys; the log-sum-exp counts them."""
    a = Attn(dtype, 5, 1, 2, 1, 7, P=1, cap=3001, lens=[[3001, 17]], kv=[1, 2, 300, 64, 77], q_scale=0.0).run().check()
    counts = torch.tensor([[[3001 + n, 17 + n]] for n in [1, 2, 300, 64, 77]], dtype=torch.float64)
    assert (a.lse.double().cpu() - counts.log()).abs().max() < 1e-5


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", ["single_row", "ragged_prompts", "chunk_333", "rows_130_g4", "long_tail"])
def test_attention_repeats_its_bits_and_needs_no_lse(name, dtype):
    a = Attn(dtype, seed=12, **CASES[name]).run()
    out, lse = a.out.clone(), a.lse.clone()
    a.run()
    assert torch.equal(out, a.out) and torch.equal(lse, a.lse)
    a.out.fill_(MARK)
    a.call(lse=False)
    assert torch.equal(out, a.out)


def _check_rows(a, rows):
    """Rows of a call that is too large for the plain form as a whole."""
    B, P = a.B, a.prefix64["K"].shape[0]
    for b in rows:
        p = ar.prompt_of(b, B, P, a.prefix64["row_start"])
        pre = None if p < 0 else dict(K=a.prefix64["K"][p:p + 1], V=a.prefix64["V"][p:p + 1], lens=a.prefix64["lens"][p:p + 1], row_start=None)
        own = dict(a.pages64, table=a.pages64["table"][b:b + 1], kv_lens=a.pages64["kv_lens"][b:b + 1])
        out, lse, bounds = ar.attention(a.q64[b:b + 1], a.G, None if a.new is None else a.new[b:b + 1], pre, own)
        o_tol, l_tol = ar.tolerance(a.dtype, out, lse, bounds)
        there = ~np.isnan(lse)
        out[~there], lse[~there], o_tol[~there], l_tol[~there] = MARK, MARK, 0.0, 0.0
        _check(a.lse[b:b + 1], lse, l_tol, f"lse of row {b}")
        _check(a.out[b:b + 1], out, o_tol, f"out of row {b}")


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_over_more_than_the_last_level_cache(dtype, page):
    """Lists so long that as many as there are of them fill half the last-level cache are read with the non-temporal hint: one such tail and two such prefixes,
    of an odd number of keys, beside short ones, which are read without."""
    _say(f"streaming {dtype} page={page}")
    B, H, esz = 8, 32, 4 if dtype == "f32" else 2
    long = (128 << 20) // (B * H * 2 * 128 * esz)              # keys a list from which on it is streamed
    lens = [[long + 37] * H, [5] * H] + [[long // 2 + p] * H for p in range(2, B)]
    lens[4] = [long + 1 if h % 2 else 0 for h in range(H)]
    kv = [40, long + 75, 2, 3, 17, 64, 1, 33]
    a = Attn(dtype, B, 2, H, 2, 20, P=B, cap=long + 37, lens=lens, kv=kv, page=page, new=[2, 2, 2, 1, 2, 0, 1, 2])
    assert gu.kernels_of(a.call) == {"prefix_attn_split_kernel", "prefix_attn_join_kernel"}
    a.run()
    _check_rows(a, range(B))


@pytest.mark.parametrize("dtype,T,G,kernel", [("f16", 1, 1, "prefix_attn_split_kernel"), ("f32", 2, 1, "prefix_attn_split_kernel"),
                                              ("bf16", 2, 40, "prefix_attn_wide_kernel"), ("f32", 2, 40, "prefix_attn_split_kernel")])
def test_more_prompts_than_a_wave_looks_through_at_once(dtype, T, G, kernel):
    """150 prompts with none to 45 rows each, rows of no prompt at both ends."""
    _say(f"many ragged prompts {dtype} T={T} G={G}")
    counts = [(7 * p) % 4 for p in range(150)]
    counts[3], counts[31], counts[32], counts[63], counts[64], counts[65], counts[100], counts[149] = 33, 0, 2, 1, 0, 45, 0, 3
    starts = (2 + np.cumsum([0] + counts)).tolist()
    B = starts[-1] + 2
    a = Attn(dtype, B, T, 1, G, 21, P=150, cap=41, lens=[[(11 * p) % 42] for p in range(150)], row_start=starts, kv=[T + (5 * b) % 23 for b in range(B)], page=8)
    assert kernel in gu.kernels_of(a.call)
    a.run()
    picked = range(B) if G == 1 else sorted({0, 1, 2, B - 1, B - 2, B - 3} | {starts[p] for p in range(0, 150, 9)} | {starts[65] + i for i in range(0, 45, 4)})
    _check_rows(a, picked)


def test_attention_beyond_32_bits():
    """Pools and prefixes of more than 2^32 elements: the last pages, the last prompt."""
    H, page, P, cap = 32, 64, 3, 400000
    n_pages = 2 ** 32 // (H * page * 128) + 3
    pool = [torch.empty((n_pages, H, page, 128), dtype=torch.float16, device="cuda") for _ in range(2)]
    pre = [torch.empty((P, H, cap, 128), dtype=torch.float16, device="cuda") for _ in range(2)]
    table, kv, lens = [[n_pages - 1, n_pages - 2], [n_pages - 3, 0]], [70, 128], [[50] * H] * P
    row_start = [0, 1, 1, 2]
    gen = torch.Generator(device="cuda").manual_seed(3)
    for t in pool:
        for p in (0, n_pages - 1, n_pages - 2, n_pages - 3):
            t[p] = torch.randn(t[p].shape, generator=gen, device="cuda").half()
    for t in pre:
        t[:, :, :50] = torch.randn((P, H, 50, 128), generator=gen, device="cuda").half()
    pages, prefix = kb.make_pages(*pool, _i32(table)), kb.make_prefix(*pre, _i32(lens), _i32(row_start))
    for T in (1, 20):
        shape = kb.make_token_shape(pages, T, 1)
        q = torch.randn((2, T, H, 128), generator=gen, device="cuda").half()
        out, lse = torch.empty_like(q), torch.empty((2, T, H), device="cuda")
        ws = torch.empty(kb.kvm_prefix_attn_workspace_bytes(shape, prefix, pages), dtype=torch.uint8, device="cuda")
        kb.kvm_prefix_attn(shape, prefix, pages, q, _i32(kv), out, lse, ws)
        host = lambda t, rows: t[rows].double().cpu().numpy()
        keep = [0, n_pages - 1, n_pages - 2, n_pages - 3]
        small = [[keep.index(p) for p in row] for row in table]
        want = ar.attention(gu.to_host_f64(q), 1, None,
                            dict(K=host(pre[0][:, :, :50], slice(None)), V=host(pre[1][:, :, :50], slice(None)), lens=None, row_start=row_start),
                            dict(K=host(pool[0], keep), V=host(pool[1], keep), table=np.array(small), kv_lens=kv))
        o_tol, l_tol = ar.tolerance("f16", *want)
        _check(out, want[0], o_tol, "out")
        _check(lse, want[1], l_tol, "lse")


# ---------------------------------------------------------------------------------------------
# streams, graphs, and the calls together
# ---------------------------------------------------------------------------------------------

def test_attention_on_two_streams_at_once():
    """Two calls with a workspace each, on two streams, several times over: the bits of the calls alone."""
    pairs = [Attn("bf16", seed=13, **CASES["ragged_prompts"]), Attn("f16", seed=14, **CASES["long_prefix"])]
    alone = [a.run().out.clone() for a in pairs]
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(3):
        torch.cuda.synchronize()
        for a in pairs:
            a.out.fill_(MARK)
        torch.cuda.synchronize()
        for a, s in zip(pairs, streams):
            with torch.cuda.stream(s):
                for _ in range(4):
                    a.call()
        torch.cuda.synchronize()
        for a, want in zip(pairs, alone):
            assert torch.equal(a.out, want)


class Answer:
    """Rows that answer compressed prompts, layer by layer as a decoding loop does it (one layer here)."""

    def __init__(self, dtype, P, rows, H, G, N, steps, page=16, seed=0, rot=64):
        self.dtype, self.P, self.H, self.G, self.steps = dtype, P, H, G, steps
        tdt = gu.TORCH_DT[dtype]
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(tdt)
        Q, K, V = normal(P, H * G, N, 128), normal(P, H, N, 128).cumsum(2).mul(0.2).to(tdt), normal(P, H, N, 128)
        lens = _i32([N - 31 * p for p in range(P)])
        cshape, params = kb.make_shape(K, G, lens), kb.kvm_params_for_budget(0.5)
        self.buf = kb.Buffers(cshape, params, "cuda", tdt)
        self.buf.K_out.fill_(float("nan"))
        self.buf.V_out.fill_(float("nan"))
        kb.compress(cshape, params, Q, K, V, self.buf)
        starts = np.cumsum([0] + rows)
        self.B = B = int(starts[-1])
        self.prefix = kb.make_prefix(self.buf.K_out, self.buf.V_out, self.buf.n_sets, _i32(starts))
        self.starts = starts
        self.table, n_pages = ar.scattered_pages(np.random.default_rng(seed), B, [steps] * B, page)
        self.Kp, self.Vp = (torch.full((n_pages, H, page, 128), float("nan"), dtype=tdt, device="cuda") for _ in range(2))
        self.pages = kb.make_pages(self.Kp, self.Vp, torch.from_numpy(self.table).cuda())
        self.shape = kb.make_token_shape(self.pages, 1, G)
        self.freq = (1.0 / 10000.0 ** (np.arange(0, rot, 2) / rot)).astype(np.float32)
        self.rotation = kb.make_rotation(torch.from_numpy(self.freq).cuda())
        self.pos = [N - 31 * p for p in range(P) for _ in range(rows[p])]
        self.pos_base = _i32(self.pos)
        self.qkv = normal(steps, B, 1, (G + 2) * H, 128)
        self.step_in = torch.empty_like(self.qkv[0])           # where a captured step finds its tokens
        self.lens = [torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2)]
        self.q_out, self.out = (torch.empty((B, 1, G * H, 128), dtype=tdt, device="cuda") for _ in range(2))
        self.ws = torch.empty(kb.kvm_prefix_attn_workspace_bytes(self.shape, self.prefix, self.pages), dtype=torch.uint8, device="cuda")

    def step(self, x, past, now):
        HG, H = self.H * self.G, self.H
        kb.kvm_paged_append(self.shape, self.pages, self.rotation, x[:, :, :HG], x[:, :, HG:HG + H], x[:, :, HG + H:], self.lens[past],
                            self.pos_base, self.q_out, self.lens[now])
        kb.kvm_prefix_attn(self.shape, self.prefix, self.pages, self.q_out, self.lens[now], self.out, None, self.ws)

    def check(self, t):
        """Step t: the stored keys, values and turned queries against the plain rotation of all inputs so far, and the output against the
        plain attention of what is stored."""
        HG, H, page = self.H * self.G, self.H, self.Kp.shape[2]
        x = self.qkv[:t + 1].double().cpu().numpy()[:, :, 0]                  # (steps, B, heads, 128)
        Kp, Vp, turned_q = gu.to_host_f64(self.Kp), gu.to_host_f64(self.Vp), gu.to_host_f64(self.q_out)
        half, rot = ar.EPS[self.dtype] / 2, 2 * len(self.freq)
        for b in range(self.B):
            for j in range(t + 1):
                got_k, got_v = Kp[self.table[b, j // page], :, j % page], Vp[self.table[b, j // page], :, j % page]
                want = ar.rotate(x[j, b, :HG + H], np.full(HG + H, self.pos[b] + j), self.freq, False)
                length = np.zeros_like(want)
                length[:, :rot] = np.tile(np.hypot(x[j, b, :HG + H, :rot // 2], x[j, b, :HG + H, rot // 2:rot]), 2)
                tol = 2.0 ** -20 * length * (1 + 2 * half) + half * np.abs(want) + ar.TINY[self.dtype]
                assert (np.abs(got_k - want[HG:]) <= tol[HG:]).all() and (got_v == x[j, b, HG + H:]).all()
                assert j < t or (np.abs(turned_q[b, 0] - want[:HG]) <= tol[:HG]).all()
        out, lse, bounds = ar.attention(turned_q, self.G, None,
                                        dict(K=gu.to_host_f64(self.buf.K_out), V=gu.to_host_f64(self.buf.V_out),
                                             lens=self.buf.n_sets.cpu().numpy(), row_start=self.starts),
                                        dict(K=Kp, V=Vp, table=self.table, kv_lens=[t + 1] * self.B))
        _check(self.out, out, ar.tolerance(self.dtype, out, lse, bounds)[0], f"step {t}")


@pytest.mark.parametrize("dtype,P,rows,H,G", [("f16", 2, [5, 9], 4, 1), ("bf16", 1, [33], 2, 4), ("f32", 3, [1, 2, 1], 2, 2)])
def test_decoding_from_a_compressed_prompt(dtype, P, rows, H, G):
    """Compression pass, then a row of steps: append and attention over the merged states and the pages."""
    _say(f"decoding {dtype} P={P} rows={rows} H={H} G={G}")
    a = Answer(dtype, P, rows, H, G, 400, 20)
    for t in range(a.steps):
        a.step(a.qkv[t], t % 2, 1 - t % 2)
        if t in (0, 7, 19):
            a.check(t)
    assert a.lens[a.steps % 2].tolist() == [a.steps] * a.B


def test_a_step_captured_into_a_graph():
    """Two captured steps (lengths go back and forth between two buffers) replayed, with eager work and synchronisation between: every
    replay has the bits of the eager loop."""
    eager = Answer("bf16", 2, [7, 4], 2, 2, 400, 12, seed=4)
    want = []
    for t in range(12):
        eager.step(eager.qkv[t], t % 2, 1 - t % 2)
        want.append(eager.out.clone())
    a = Answer("bf16", 2, [7, 4], 2, 2, 400, 12, seed=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                              # once outside, as a program warms up
        a.step_in.copy_(a.qkv[0])
        a.step(a.step_in, 0, 1)
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            a.step(a.step_in, i, 1 - i)
    for n in a.lens:
        n.zero_()
    for t in range(12):
        a.step_in.copy_(a.qkv[t])
        graphs[t % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[t]), t
        eager.step(eager.qkv[0], 0, 1)                         # eager work of the program between the replays


def test_argument_checks_of_the_binding():
    a = Attn("f16", seed=1, **CASES["drafts"])
    bad = lambda **kw: dict(dict(shape=a.shape, prefix=a.prefix, pages=a.pages, Q=a.q, kv_lens=a.kv_lens, out=a.out, lse_opt=a.lse, ws=a.ws), **kw)
    for kw in (dict(Q=a.q.float()), dict(Q=a.q[:, :2]), dict(out=a.out.transpose(0, 1)), dict(kv_lens=a.kv_lens.long()), dict(kv_lens=a.kv_lens[:3]),
               dict(lse_opt=a.lse[:2]), dict(lse_opt=a.lse.half()), dict(Q=a.q.cpu()), dict(out=a.out[..., :64])):
        with pytest.raises(ValueError):
            kb.kvm_prefix_attn(**bad(**kw))
    with pytest.raises(kb.KvmError):
        kb.kvm_prefix_attn(**bad(ws=a.ws[:16]))
    with pytest.raises(ValueError):                            # rows of another batch
        kb.kvm_prefix_attn(**bad(shape=kb.make_token_shape(a.prefix, 3, 2, None, B=9)))
    with pytest.raises(ValueError):
        kb.make_token_shape(a.pages, 3, 2, torch.ones(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        kb.make_prefix(a.prefix._refs[0], a.prefix._refs[1], torch.ones((3, 2), dtype=torch.int32, device="cuda"))
