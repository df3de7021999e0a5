"""The serving step's operators on the GPU against their definitions in 64 bits.

Tolerances, from the roundings made (u = half a step of the type, f = 2^-24):
  attention  one rounding of the output, u |o|; every weight is rounded to the type once, u A with A = sum w |v| (fp16 weights also stand at least
             2^-31 of the greatest apart: part of the term below); scores are sums of D products in 32 bits, then multiplied and subtracted in 32 bits, so
             a weight is off by d = (D + 8) f S + 2^-20 with S the greatest sum of |q k| scale of the row, in the numerator and in the sum: 2 d A; the
             sums over n keys in 32 bits, 2 n f A at most
  append     one rounding of the output, u |x|; sine and cosine to 2^-20 (angle fraction of a turn rounded to 32 bits, functions good to 2 f)
  8 bits     half a step, 2^-4 relative or 2^-10 below 2^-6, of value / scale
"""
import numpy as np
import pytest
import torch

from tests import serve_plain as plain

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F = 2.0 ** -24
E4M3 = torch.float8_e4m3fn
FIT = "8 bits that hold every value"      # with plain E4M3 some of a Cache's values are beyond what the type holds: NaN


def _dyn():
    import paper_2408_00741_amd as dyn
    return dyn


def _np(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _close(got, want, tol, what=""):
    got = _np(got).astype(np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    off = np.abs(got - want)[fine] - np.broadcast_to(tol, want.shape)[fine]
    assert off.size == 0 or off.max() <= 0, f"{what}: {off.max()} beyond the tolerance, {np.mean(off > 0)} of the values"


class Cache:
    """Requests with lengths, a block table over shuffled pages, and a cache filled with normal values (unused rows with `fill`)."""

    def __init__(self, new, kv, G, D, P, dtype, cache=None, seed=0, fill=float("nan"), extra=3):
        g = torch.Generator().manual_seed(seed)
        self.new, self.kv = np.asarray(new), np.asarray(kv)
        pages = -(-self.kv // P)
        self.N, cols = int(pages.sum()) + extra, max(1, int(pages.max())) + 1
        order = torch.randperm(self.N, generator=g).numpy().astype(np.int32)
        self.table = np.full((len(kv), cols), -1, np.int32)
        at = 0
        for b, p in enumerate(pages):
            self.table[b, :p] = order[at:at + p]
            at += p
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.k_scale = self.v_scale = None
        cache = cache or dtype
        fit = cache == FIT
        cache = E4M3 if fit else cache
        if cache == E4M3:
            self.k_scale, self.v_scale = (torch.rand(G, generator=g) * 0.02 + 0.005 for _ in range(2))
        used = np.zeros((self.N, P), bool)
        for b, L in enumerate(self.kv):
            for i in range(-(-int(L) // P)):
                used[self.table[b, i], :min(P, int(L) - i * P)] = True
        m = torch.from_numpy(used)[:, None, :, None]

        def one(scale):
            x = torch.randn(self.N, G, P, D, generator=g)
            if scale is not None:
                x = x / scale[:, None, None]
                x = x.clamp(-448, 448) if fit else x
            return torch.where(m, x, torch.full((), fill)).to(cache)
        self.k, self.v = one(self.k_scale), one(self.v_scale)
        self.G, self.D, self.P, self.dtype = G, D, P, dtype
        self.g = g

    def queries(self, H, factor=2.0):
        return (factor * torch.randn(int(self.cu[-1]), H, self.D, generator=self.g)).to(self.dtype)

    def run(self, q, workspace=None, **kw):
        c = lambda x: None if x is None else (torch.from_numpy(x) if isinstance(x, np.ndarray) else x).cuda()  # noqa: E731
        i = lambda a: c(np.asarray(a, np.int32))  # noqa: E731
        kw.setdefault("max_new", int(self.new.max()))
        kw.setdefault("max_kv", int(self.kv.max()))
        out = _dyn().dyn_paged_attention(q if q.is_cuda else q.cuda(), c(self.k), c(self.v), i(self.table), i(self.cu), i(self.kv), k_scale=c(self.k_scale),
                                         v_scale=c(self.v_scale), workspace=workspace, **kw)
        torch.cuda.synchronize()
        return out

    def check(self, q, out, scale=None, window=0, n_sink=0):
        scale = self.D ** -0.5 if scale is None else scale
        # the factor reaches the kernel in 32 bits
        want, size, score = plain.attention(_np(q), _np(self.k), _np(self.v), self.table, self.cu, self.kv, float(np.float32(scale)), window, n_sink,
                                            None if self.k_scale is None else _np(self.k_scale), None if self.v_scale is None else _np(self.v_scale))
        u = U[self.dtype]
        d = (self.D + 8) * F * score[..., None] + 2.0 ** -20
        with np.errstate(invalid="ignore"):
            _close(out, want, u * np.abs(want) + (u + 2 * d + 2 * F * float(self.kv.max())) * size + 1e-30)


TYPES = [(torch.bfloat16, None), (torch.float16, None), (torch.bfloat16, E4M3), (torch.float16, E4M3), (torch.bfloat16, FIT), (torch.float16, FIT)]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("lens", [[1], [2, 1, 31], [32, 33, 64, 65], [127, 128, 129, 500, 7]])
def test_attention_single_tokens(dtype, cache, lens):
    c = Cache([1] * len(lens), lens, 2, 128, 16, dtype, cache, seed=len(lens))
    q = c.queries(16)
    c.check(q, c.run(q))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D,G,group,P", [(16, 1, 1, 1), (48, 3, 5, 4), (64, 2, 8, 32), (80, 2, 3, 16), (112, 1, 32, 128), (128, 1, 40, 4096), (96, 4, 1, 64)])
def test_attention_heads_and_pages(dtype, cache, D, G, group, P):
    c = Cache([1, 1, 3, 40], [70, 1, 333, 200], G, D, P, dtype, cache, seed=D)
    q = c.queries(G * group)
    c.check(q, c.run(q))


@pytest.mark.parametrize("dtype,cache", TYPES[:3] + TYPES[4:5])
@pytest.mark.parametrize("new,kv", [([1, 17, 63, 129, 300], [1, 17, 100, 129, 777]),          # from the start, and over a context
                                    ([64, 0, 5, 33, 1], [64, 50, 3, 0, 0]),                      # no new tokens; fewer keys than tokens; none
                                    ([257], [1025]), ([2, 2, 2], [2, 1, 0])])
def test_attention_chunks(dtype, cache, new, kv):
    c = Cache(new, kv, 2, 64, 16, dtype, cache, seed=sum(new))
    q = c.queries(8)
    c.check(q, c.run(q))


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 1), (64, 4), (100, 70), (33, 0), (1000, 5), (40, 1000)])
@pytest.mark.parametrize("new,kv", [([1, 1, 1], [1, 90, 700]), ([130, 9, 1], [400, 9, 333])])
def test_attention_window(window, sinks, new, kv):
    c = Cache(new, kv, 2, 64, 16, torch.bfloat16, seed=window)
    q = c.queries(8)
    c.check(q, c.run(q, window=window, n_sink=sinks), window=window, n_sink=sinks)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("new,kv", [([1, 1], [9001, 130]), ([3], [5000]), ([70], [4000])])
def test_attention_long_cut_in_pieces(dtype, cache, new, kv):
    c = Cache(new, kv, 1, 128, 32, dtype, cache, seed=11)
    q = c.queries(4)
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    out = c.run(q, workspace=ws)
    c.check(q, out)
    assert _dyn().dyn_workspace_status(ws) == 0
    again = c.run(q, workspace=ws)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))   # the same bits on every run


@pytest.mark.parametrize("new,kv,D,G,group,window,n_sink", [
    ([300, 1, 20, 419], [2000, 500, 1900, 2100], 16, 6, 16, 0, 0),      # 540 pairs of a row tile and a key head: full rounds of whole ones, the others cut
    ([0, 700, 3, 40], [0, 2100, 40, 1990], 64, 3, 32, 1500, 9),         # the same under a window, with numbers that have no row tile
    ([500], [500], 48, 8, 16, 0, 0),                                    # a prompt from its start: nothing is cut
    ([200, 60], [260, 333], 16, 32, 32, 0, 0),                          # more pairs than are dealt out: a block is one
    ([40, 33], [40, 333], 32, 2, 4, 0, 0)])                             # no request of few rows can be there: none is looked for
def test_attention_row_tiles_dealt_out(new, kv, D, G, group, window, n_sink):
    c = Cache(new, kv, G, D, 16, torch.bfloat16, seed=D)
    q = c.queries(G * group)
    out = c.run(q, window=window, n_sink=n_sink)
    c.check(q, out, window=window, n_sink=n_sink)
    assert torch.equal(out, c.run(q, window=window, n_sink=n_sink))


def test_attention_fewer_tokens_than_rows_of_the_tensor():
    # a captured step has room for more tokens than a step brings: one request of one token in a tensor of 64
    c = Cache([1], [100], 2, 64, 16, torch.float16, seed=9)
    q = torch.cat([c.queries(8), torch.zeros(63, 8, 64, dtype=torch.float16)])
    for most in (1, 64):
        out = c.run(q, max_new=most)
        c.check(q[:1], out[:1])


def test_attention_workspace_is_shared_by_calls_of_other_shapes():
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    for i, (new, kv, G) in enumerate([([1, 1], [3000, 200], 1), ([90], [2500], 2), ([1] * 40, [64] * 40, 4), ([1], [5000], 1), ([200, 1], [1500, 900], 1)]):
        c = Cache(new, kv, G, 64, 16, torch.bfloat16, seed=i)
        q = c.queries(4 * G)
        c.check(q, c.run(q, workspace=ws))


@pytest.mark.parametrize("scale", [-0.11, 0.0, 3.0])
def test_attention_scales(scale):
    c = Cache([1, 40], [300, 100], 2, 64, 16, torch.float16, seed=4)
    q = c.queries(8, 1.0)
    c.check(q, c.run(q, scale=scale), scale=scale)
    c = Cache([1, 40], [300, 100], 2, 64, 16, torch.bfloat16, E4M3, seed=4)
    c.k_scale[0], c.k_scale[1], c.v_scale[0] = 0.0, -0.01, -0.02
    q = c.queries(8, 1.0)
    c.check(q, c.run(q, scale=scale), scale=scale)
    c = Cache([1, 40], [300, 100], 2, 64, 16, torch.bfloat16, FIT, seed=4)
    c.k_scale[0], c.k_scale[1], c.v_scale[0] = 0.0, -0.01, -0.02
    q = c.queries(8, 1.0)
    c.check(q, c.run(q, scale=scale), scale=scale)


@pytest.mark.parametrize("new,kv", [([1, 1], [50, 700]), ([150], [333])])
def test_attention_far_apart_scores(new, kv):
    # scores of hundreds: one key takes all, the others' weights pass below what the types hold; the maximum rises late
    for dtype in U:
        c = Cache(new, kv, 1, 128, 16, dtype, seed=8)
        c.k[c.table[0, int(c.kv[0] - 1) // 16], 0, int(c.kv[0] - 1) % 16] *= 8
        q = c.queries(8, 6.0)
        c.check(q, c.run(q))


@pytest.mark.parametrize("offset,gap", [(0, 8), (1, 3), (4, 4)])
@pytest.mark.parametrize("new,kv", [([1, 1], [50, 700]), ([150, 1], [333, 20])])
def test_attention_strides(offset, gap, new, kv):
    c = Cache(new, kv, 2, 64, 16, torch.bfloat16, seed=3)
    q = c.queries(8)
    T = q.shape[0]
    room = torch.full((T * 8 * (64 + gap) + 64,), float("nan"), dtype=q.dtype, device="cuda")
    qs = room[offset:offset + T * 8 * (64 + gap)].view(T, 8, 64 + gap)[..., :64]
    qs.copy_(q)
    hold = torch.full((8, T, 64 + gap), 7.0, dtype=q.dtype, device="cuda")                       # heads before tokens
    out = hold.transpose(0, 1)[..., :64]
    c.run(qs, out=out)
    c.check(q, out)
    assert torch.all(hold[..., 64:] == 7.0)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", list(U))
@pytest.mark.parametrize("window", [0, 20])
def test_attention_not_finite_where_hidden_and_where_seen(bad, dtype, window):
    c = Cache([1, 70, 40], [100, 90, 300], 2, 64, 16, dtype, seed=5)
    at = lambda b, x: (c.table[b, x // 16], slice(None), x % 16)  # noqa: E731
    c.v[at(1, 60)][0, 5] = bad                                      # seen by the later tokens of request 1 only
    c.v[at(1, 61)][1, 63] = -bad
    c.k[at(1, 80)] = float("nan")                                   # hidden from all before it
    c.v[at(2, 10)] = bad                                            # far before the window
    c.v[at(0, 99)][0, 0] = bad                                      # a single token's own value
    q = c.queries(8)
    c.check(q, c.run(q, window=window), window=window)


def test_attention_page_outside_the_cache():
    dyn = _dyn()
    c = Cache([1, 1], [100, 200], 2, 64, 16, torch.bfloat16, seed=6)
    q = c.queries(8)
    good = c.run(q)
    for wrong in (-7, c.N, 1 << 30):
        keep = c.table[0, 2]
        c.table[0, 2] = wrong
        ws = torch.zeros(32 << 20, dtype=torch.uint8, device="cuda")
        out = c.run(q, workspace=ws)
        assert dyn.dyn_workspace_status(ws) == dyn.DYN_WS_BAD_PAGE
        assert torch.equal(out[1], good[1])                        # the other request's row
        c.table[0, 2] = keep


def test_attention_on_another_stream():
    c = Cache([1, 80], [600, 200], 2, 128, 16, torch.bfloat16, seed=9)
    q = c.queries(8)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out = c.run(q)
    c.check(q, out)
    out = c.run(q, stream=s)
    c.check(q, out)


def test_attention_cache_beyond_32_bits():
    # pages at the end of a cache whose byte offsets need more than 32 bits
    N, G, P, D = 70_000, 8, 32, 128
    k = torch.empty(N, G, P, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() * 2 > 1 << 32
    c = Cache([1, 70], [300, 90], G, D, P, torch.bfloat16, seed=2)
    here = torch.arange(c.N) + N - c.N
    k[here] = c.k.cuda()
    v[here] = c.v.cuda()
    q = c.queries(8)
    t = torch.from_numpy(c.table + (N - c.N)).cuda()
    i = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
    out = _dyn().dyn_paged_attention(q.cuda(), k, v, t, i(c.cu), i(c.kv), 70, 300)
    c.check(q, out)


# ---- rotary positions and the cache's new rows -------------------------------------------------------------------

def _append(T, H, G, D, P, N, dtype, cache, rotary, interleaved, seed, amplitude=1.0, scaled=True, gap=0, offset=0, far=False):
    dyn, g = _dyn(), torch.Generator().manual_seed(seed)
    hold = torch.randn(T * (H + 2 * G) * (D + gap) + 8, generator=g).to(dtype).cuda()
    qkv = hold[offset:offset + T * (H + 2 * G) * (D + gap)].view(T, H + 2 * G, D + gap)[..., :D]
    q, k, v = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    pos = torch.randint(0, 1 << 30 if far else 5000, (T,), generator=g).to(torch.int32)
    slot = torch.randperm(N * P, generator=g)[:T].to(torch.int32)
    if T > 2:
        slot[1], pos[1] = -1, -1
        slot[2] = N * P + 5
    w, _ = dyn.dyn_rope_frequencies(rotary) if rotary else (np.empty(0), 1.0)
    ks, vs = ((torch.rand(G, generator=g) + 0.5) * 0.02 if cache == E4M3 and scaled else None for _ in range(2))
    before = [torch.randn(N, G, P, D, generator=g).to(cache) for _ in range(2)]
    kc, vc = (x.cuda() for x in before)
    cu = lambda x: None if x is None else x.cuda()  # noqa: E731
    out = dyn.dyn_rope_append(q, k, v, pos.cuda(), slot.cuda(), kc, vc, w, interleaved=interleaved, rope_scale=amplitude, k_scale=cu(ks), v_scale=cu(vs))
    u = U[dtype]
    amp = float(np.float32(amplitude))
    turned = lambda x: plain.rotate(_np(x), pos.numpy(), w, interleaved, amp)  # noqa: E731
    # the other element of a pair counts with what sine and cosine may be off
    sizes = lambda x: np.abs(_np(x)).max(-1, keepdims=True) * (abs(amp) + 1.0) * 2.0 ** -20 if rotary else 0.0  # noqa: E731
    want = turned(q)
    _close(out, want, u * np.abs(want) + sizes(q), "q")
    for name, x, got, was, f in (("k", turned(k), kc, before[0], ks), ("v", _np(v).astype(np.float64), vc, before[1], vs)):
        want = _np(was).astype(np.float64)
        tol = np.zeros_like(want)
        slack = sizes(k) if name == "k" else np.zeros((T, G, 1))
        for t in range(T):
            s = int(slot[t])
            if 0 <= s < N * P:
                y = x[t] if f is None else np.clip(x[t] / _np(f).astype(np.float64)[:, None], -448, 448)
                sl = (slack[t] if rotary else 0.0) if f is None else slack[t] / _np(f).astype(np.float64)[:, None] if rotary else 0.0
                if cache == E4M3:
                    if f is None:
                        y = np.clip(y, -448, 448)
                    e = np.maximum(2.0 ** -10, 2.0 ** -4 * np.abs(y)) + sl * 1.1 + 4 * F * np.abs(y)
                else:
                    e = u * np.abs(y) + sl
                want[s // P, :, s % P], tol[s // P, :, s % P] = y, e
        _close(got, want, tol, name)


@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, E4M3), (torch.float16, E4M3)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rotary", [(128, 128), (128, 64), (80, 40), (64, 6), (16, 2), (96, 0), (112, 112)])
def test_append_layouts(dtype, cache, interleaved, D, rotary):
    _append(19, 6, 2, D, 16, 7, dtype, cache, rotary, interleaved, seed=D + rotary)


@pytest.mark.parametrize("gap,offset", [(8, 0), (4, 4), (1, 0), (0, 1)])
def test_append_strides(gap, offset):
    _append(9, 4, 1, 64, 8, 5, torch.float16, torch.float16, 64, False, seed=gap, gap=gap, offset=offset)
    _append(9, 4, 1, 64, 8, 5, torch.bfloat16, E4M3, 32, True, seed=gap, gap=gap, offset=offset, scaled=False)


def test_append_one_token_many_tokens_and_far_positions():
    _append(1, 64, 8, 128, 16, 2, torch.bfloat16, torch.bfloat16, 128, False, seed=1)
    _append(2100, 2, 1, 32, 16, 200, torch.bfloat16, torch.bfloat16, 32, True, seed=2, amplitude=1.37)
    _append(33, 2, 1, 64, 1, 64, torch.float16, torch.float16, 64, False, seed=3, far=True)


def test_append_values_that_8_bits_cannot_hold():
    dyn = _dyn()
    x = torch.tensor([0.0, 1.0, -1.0, 447.0, 460.0, 465.0, -1e4, float("inf"), -float("inf"), float("nan"), 2.0 ** -10, 2.0 ** -9 * 1.5, 3e-5, 17.0, 18.0, 19.0])
    q = torch.zeros(1, 1, 16, dtype=torch.float16, device="cuda")
    k = x.to(torch.float16).view(1, 1, 16).cuda()
    kc, vc = (torch.zeros(1, 1, 1, 16, dtype=E4M3, device="cuda") for _ in range(2))
    z = torch.zeros(1, dtype=torch.int32, device="cuda")
    dyn.dyn_rope_append(q, k, k, z, z, kc, vc, np.empty(0))
    want = k.float().clamp(-448, 448).cpu().view(-1)
    want = torch.where(torch.isnan(k.float().cpu().view(-1)), torch.full((), float("nan")), want).to(E4M3).float().numpy()
    for got in (kc, vc):
        assert np.array_equal(got.float().cpu().numpy().reshape(-1), want, equal_nan=True)


# ---- block tables and slot maps -----------------------------------------------------------------------------------

def _requests(B, page, seed, room=2.0, context=300, chunk=40, released=0.1, max_pages=None):
    r = np.random.RandomState(seed)
    ctx = r.randint(0, context, B).astype(np.int32)
    new = np.where(r.rand(B) < 0.5, 1, r.randint(0, chunk, B)).astype(np.int32)
    new[r.rand(B) < released] = -1
    have = -(-ctx // page)
    cols = max_pages or int((-(-(ctx + np.maximum(new, 0)) // page)).max()) + 2
    ctx = np.minimum(ctx, cols * page).astype(np.int32)
    have = -(-ctx // page)
    ask = int((-(-(ctx + np.maximum(new, 0)) // page) - have).sum())
    free = int(ask * room) + 1
    N = int(have.sum()) + free
    pool = r.permutation(N).astype(np.int32)
    table = np.full((B, cols), -1, np.int32)
    at = 0
    for b, h in enumerate(have):
        table[b, :h] = pool[at:at + h]
        at += h
    first = int(r.randint(0, N))
    ring = np.zeros(N, np.int32)
    ring[(first + np.arange(free)) % N] = pool[at:]
    return ctx, new, table, ring, np.array([first, free], np.int32)


def _check_step(ctx, new, table, ring, state, page):
    dyn = _dyn()
    T = int(np.maximum(new, 0).sum())
    c = lambda a: torch.from_numpy(a.copy()).cuda()  # noqa: E731
    p = dyn.dyn_kv_step(c(ctx), c(new), T, c(table), c(ring), c(state), page)
    want = plain.step(ctx, new, table, ring, state, page, T)
    for name, w in zip(("cu_new", "kv_len", "next_len", "pos", "slot", "block_table", "free_pages", "free_state"), want):
        assert np.array_equal(p[name].cpu().numpy(), w), name
    assert dyn.dyn_workspace_status(p.workspace) == (dyn.DYN_WS_NO_PAGES if any(want[-1]) else 0)
    return p


@pytest.mark.parametrize("page", [1, 16, 256])
@pytest.mark.parametrize("B", [1, 3, 64, 255, 256, 257, 1000, 2047, 2048, 2049, 5000])
def test_step(B, page):
    _check_step(*_requests(B, page, seed=B + page), page)


@pytest.mark.parametrize("B,room,cols", [(50, 0.5, None), (50, 0.0, None), (3000, 0.7, None), (300, 2.0, 12), (2500, 2.0, 12)])
def test_step_refuses(B, room, cols):
    _check_step(*_requests(B, 16, seed=B, room=room, max_pages=cols), 16)


def test_step_of_no_tokens_and_of_many():
    ctx, new, table, ring, state = _requests(40, 16, seed=1)
    _check_step(ctx, np.zeros_like(new), table, ring, state, 16)
    _check_step(ctx, np.full_like(new, -1), table, ring, state, 16)
    _check_step(*_requests(7, 8, seed=2, chunk=30000, context=20000), 8)


def test_step_after_step():
    # a run of steps hands out what was given back, without a page twice
    page = 4
    ctx, new, table, ring, state = _requests(30, page, seed=3, room=1.0)
    r = np.random.RandomState(5)
    for _ in range(25):
        p = _check_step(ctx, new, table, ring, state, page)
        ctx, table, ring, state = (p[k].cpu().numpy() for k in ("next_len", "block_table", "free_pages", "free_state"))
        held = np.concatenate([table[b, :-(-ctx[b] // page)] for b in range(len(ctx))])
        free = ring[(state[0] + np.arange(state[1])) % ring.size]
        assert np.array_equal(np.sort(np.concatenate([held, free])), np.arange(ring.size))
        new = np.where(r.rand(30) < 0.2, -1, r.randint(0, 9, 30)).astype(np.int32)


def test_step_with_lengths_that_cannot_be():
    dyn = _dyn()
    ctx, new, table, ring, state = _requests(20, 16, seed=4, released=0.0)
    c = lambda a: torch.from_numpy(a.copy()).cuda()  # noqa: E731
    T = int(np.maximum(new, 0).sum())
    for B in (20, 2100):
        for k, (cx, nw, t) in {"ctx": (-5, 1, T), "long": (1 << 30, 1, T), "new": (3, -9, T), "sum": (3, 2, T + 40), "less": (3, 2, max(1, T - 40)), "huge": (3, 2 ** 31 - 1, T)}.items():
            a, n = np.resize(ctx, B).astype(np.int32), np.resize(new, B).astype(np.int32)
            a[4], n[4] = cx, nw
            tab = np.resize(table, (B, table.shape[1])).astype(np.int32)
            p = dyn.dyn_kv_step(c(a), c(n), t, c(tab), c(ring), c(state), 16)
            assert dyn.dyn_workspace_status(p.workspace) & dyn.DYN_WS_BAD_REQUEST, (B, k)
            slot = p["slot"].cpu().numpy()
            assert slot.min() >= -1 and slot.max() < ring.size * 16
            cu = p["cu_new"].cpu().numpy()
            assert np.all(np.diff(cu) >= 0) and cu[-1] <= t
    bad = np.array([-3, 10 ** 6], np.int32)
    p = dyn.dyn_kv_step(c(ctx), c(new), T, c(table), c(ring), c(bad), 16)
    assert dyn.dyn_workspace_status(p.workspace) & dyn.DYN_WS_BAD_PAGE


# ---- the three together --------------------------------------------------------------------------------------------

def test_steps_of_a_server_and_their_graph():
    """Prompts in chunks beside single tokens, step after step; the step captured once and replayed with other lengths gives what eager calls give."""
    dyn = _dyn()
    B, H, G, D, P, N, cols, T = 5, 8, 2, 64, 16, 80, 16, 24
    g = torch.Generator().manual_seed(0)
    w, amp = dyn.dyn_rope_frequencies(D, scaling=dyn.DYN_ROPE_PARTS, factor=4.0, original_tokens=64.0)
    dev = "cuda"
    k1, v1 = (torch.zeros(N, G, P, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
    k2, v2 = torch.zeros_like(k1), torch.zeros_like(v1)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=dev)  # noqa: E731
    s = {"ctx": i32([0] * B), "new": i32([0] * B), "table": torch.full((B, cols), -1, dtype=torch.int32, device=dev), "ring": torch.arange(N, dtype=torch.int32, device=dev),
         "state": i32([3, N]), "qkv": torch.zeros(T, H + 2 * G, D, dtype=torch.bfloat16, device=dev), "ws": torch.zeros(32 << 20, dtype=torch.uint8, device=dev)}

    def step(s, k, v):
        p = dyn.dyn_kv_step(s["ctx"], s["new"], T, s["table"], s["ring"], s["state"], P)
        q, kk, vv = s["qkv"][:, :H], s["qkv"][:, H:H + G], s["qkv"][:, H + G:]
        q = dyn.dyn_rope_append(q, kk, vv, p["pos"], p["slot"], k, v, w, rope_scale=amp)
        o = torch.zeros(T, H, D, dtype=torch.bfloat16, device=dev)
        dyn.dyn_paged_attention(q, k, v, s["table"], p["cu_new"], p["kv_len"], T, cols * P, workspace=s["ws"], out=o)
        return p, o

    e = {x: t.clone() for x, t in s.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step({x: t.clone() for x, t in s.items()}, k2.clone(), v2.clone())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p, o = step(s, k2, v2)
    for new in ([9, 1, 14, 0, 0], [1, 1, 1, 20, 1], [1, 7, 1, 1, 1], [-1, 1, 1, 1, 1], [12, 1, -1, 1, 1], [1, 1, 15, 1, 1], [1, 1, 1, 1, 1]):
        qkv = torch.randn(T, H + 2 * G, D, generator=g).to(torch.bfloat16)
        for x in (s, e):
            x["new"].copy_(i32(new))
            x["qkv"].copy_(qkv)
        graph.replay()
        pe, oe = step(e, k1, v1)
        torch.cuda.synchronize()
        n = int(pe["cu_new"][-1])
        assert torch.equal(o, oe) and torch.equal(k1, k2) and torch.equal(v1, v2) and torch.equal(s["table"], e["table"])
        assert torch.equal(p["slot"][:n], pe["slot"][:n])
        # against the definition
        table, cu, kv = e["table"].cpu().numpy(), pe["cu_new"].cpu().numpy(), pe["kv_len"].cpu().numpy()
        q = dyn.dyn_rope_append(e["qkv"][:, :H], e["qkv"][:, H:H + G], e["qkv"][:, H + G:], pe["pos"], torch.full_like(pe["slot"], -1), k1, v1, w, rope_scale=amp)
        want, size, score = plain.attention(_np(q), _np(k1), _np(v1), table, cu, kv, float(np.float32(D ** -0.5)))
        u = U[torch.bfloat16]
        _close(oe[:n], want[:n], (u * np.abs(want) + (u + 2 * ((D + 8) * F * score[..., None] + 2.0 ** -20) + 1e-4) * size)[:n] + 1e-30)
        for x, pp in ((s, p), (e, pe)):
            x["ctx"].copy_(pp["next_len"])
            x["state"].copy_(pp["free_state"])
