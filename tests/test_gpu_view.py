"""Attention over a bounded view of the prefix (window and sinks, 4-bit cache) against
the float64 oracle.

Tolerances.  In bf16 a probability and the output are rounded once each, by at most
half a step, 2^-8 of the value; scores, maxima and sums are float32, whose part is
below 1e-3 of a probability at these sizes (128 products of up to |q k| scale = 40
in 2^-24 each).  So |O - ref| <= (2^-8 + 1e-3) A + 2^-8 |ref| with A = sum p |v|; and
the log-sum-exp is within 1e-4 + 2^-22 |ref|.  In float32 the scores' part is all:
1e-4 A, and the same for the log-sum-exp.
"""

import numpy as np
import pytest
import torch

import oracle
import paper_2609_19868_amd as Z
import workloads as W
from gpu_helpers import require_gpu, say, to_dev

pytestmark = pytest.mark.gpu


def check(out, lse, ref, dtype, what=""):
    O, L, A = ref
    got = out.float().cpu().numpy().astype(np.float64)
    nan = np.isnan(O)
    assert np.array_equal(np.isnan(got), nan), f"{what}: {np.isnan(got).sum()} NaN, {nan.sum()} expected"
    half = 2.0 ** -8
    bound = (half + 1e-3) * A + half * np.abs(O) if dtype == "bf16" else 1e-4 * A
    with np.errstate(invalid="ignore"):
        bad = (np.abs(got - O) > bound + 1e-30) & ~nan
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outputs off, first at {np.argwhere(bad)[0]}"
    le = np.abs(lse.cpu().numpy().astype(np.float64) - L)
    assert np.nanmax(le - 2.0 ** -22 * np.abs(L)) <= 1e-4, f"{what}: log-sum-exp off by {np.nanmax(le):.3e}"


class Case:
    """Seeded inputs of one call, on the host in float64 and on the device."""

    def __init__(self, dev, B, heads, D, P, S, L, dtype="bf16", cap=0, q4=False, lens=None, seed=1, q_scale=1.0,
                 slot_pass=None, **how):
        wl = W.WORKLOADS["qwen0.6b"].replace(batch=B, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=D, prefix_len=P,
                                             n_slots=S, slot_len=L, dtype=dtype, kv_capacity=P + cap, seed=seed)
        x = W.attention_inputs(wl, q_scale=q_scale)
        self.dev, self.wl, self.dtype, self.q4, self.how = dev, wl, dtype, q4, how
        self.f = {k: W.as_f64(v, dtype) for k, v in x.items()}
        self.d = {k: to_dev(v, dtype, dev) for k, v in x.items()}
        self.lens = lens
        self.clamped = P if lens is None else [min(max(n, 0), P) for n in lens]
        self.slot_pass = None
        if slot_pass:
            rng = np.random.default_rng(seed)
            self.slot_pass = rng.integers(0, 2, (B, S)).astype(np.uint8)
        if q4:
            self.codes = oracle.q4_quantize(self.f["k_cache"]) + oracle.q4_quantize(self.f["v_cache"])
            self.f["k_cache"] = oracle.q4_dequantize(*self.codes[:2])
            self.f["v_cache"] = oracle.q4_dequantize(*self.codes[2:])
            self.cache = Z.Q4Cache(*(torch.from_numpy(c).to(dev) for c in self.codes))

    def run(self, **more):
        wl, d = self.wl, self.d
        kw = dict(self.how, **more)
        if self.lens is not None:
            kw["prefix_lens"] = torch.tensor(self.lens, dtype=torch.int32, device=self.dev)
        if self.slot_pass is not None:
            kw["slot_pass"] = torch.from_numpy(self.slot_pass).to(self.dev)
        kw["prefix_len"] = wl.prefix_len
        if self.q4:
            r = Z.slot_attn_q4(d["q"], self.cache, d["k_slot"], d["v_slot"], wl.n_slots, wl.slot_len, **kw)
        else:
            r = Z.slot_attn(d["q"], d["k_cache"], d["v_cache"], d["k_slot"], d["v_slot"], wl.n_slots, wl.slot_len, **kw)
        torch.cuda.synchronize()
        return r

    def ref(self):
        wl, f, h = self.wl, self.f, self.how
        return oracle.view_attention(f["q"], f["k_cache"], f["v_cache"], f["k_slot"], f["v_slot"], self.clamped,
                                     wl.n_slots, wl.slot_len, wl.scale, h.get("pass_", 0), h.get("cross_slot", 0),
                                     self.slot_pass, h.get("window"), h.get("sinks", 0))


# (heads, S, L): 1, 4, 14, 17, 32, 33, 96, 128 and 260 rows a group, each of which
# takes another block or leaves part of one empty
ROWS = [((2, 2), 1, 1), ((8, 2), 1, 1), ((7, 1), 1, 2), ((1, 1), 17, 1), ((4, 1), 2, 4), ((3, 1), 1, 11), ((2, 1), 6, 8),
        ((4, 2), 8, 8), ((4, 1), 5, 13)]


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("heads,S,L", ROWS)
def test_rows_of_every_block(heads, S, L, q4, dtype, D):
    dev = require_gpu()
    for i, (P, window, sinks) in enumerate([(0, 3, 2), (1, 1, 0), (70, None, 0), (70, 33, 4), (333, 64, 65), (333, 500, 1)]):
        if window is None and not q4:
            window = 10 ** 6
        say(f"rows {heads} {S}x{L} q4={q4} {dtype} D={D} P={P} window={window} sinks={sinks}")
        c = Case(dev, 2, heads, D, P, S, L, dtype, cap=i, q4=q4, seed=10 + i, pass_=i % 2, cross_slot=i // 2 % 2,
                 window=window, sinks=sinks)
        check(*c.run(), c.ref(), dtype, f"P={P} window={window}")


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("heads,S,L", [((4, 2), 1, 1), ((4, 2), 8, 8)])
@pytest.mark.parametrize("splits", [0, 1, 3, 64])
def test_ragged_prefixes_and_splits(splits, heads, S, L, q4):
    """Prefixes of no row, of one, at and around a tile's end, and lengths out of range."""
    dev = require_gpu()
    lens = [0, 1, 31, 32, 33, 63, 64, 65, 700, 999, -5, 5000]
    for window, sinks in [(None, 0), (40, 3), (640, 130), (1, 0), (2 ** 31 - 1, 2 ** 31 - 1)]:
        if window is None and not q4:
            continue
        say(f"ragged splits={splits} {heads} {S}x{L} q4={q4} window={window} sinks={sinks}")
        c = Case(dev, len(lens), heads, 128, 999, S, L, cap=1, q4=q4, lens=lens, seed=3, q_scale=4.0, slot_pass=True,
                 window=window, sinks=sinks, prefix_splits=splits)
        check(*c.run(), c.ref(), "bf16", f"window={window} sinks={sinks}")


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(9, 0), (64, 4), (100, 200)])
def test_causal_layout(window, sinks, dtype, q4):
    """Many draft tokens in a causal order, the sinks partly or wholly among them."""
    dev = require_gpu()
    for P, per_slot in [(0, False), (3, True), (150, False)]:
        if q4 and not P:
            continue
        say(f"layout q4={q4} {dtype} window={window} sinks={sinks} P={P}")
        c = Case(dev, 1, (4, 2), 64, P, 24, 9, dtype, q4=q4, seed=5, slot_pass=per_slot, pass_=1, cross_slot=1,
                 window=window, sinks=sinks)
        check(*c.run(), c.ref(), dtype, f"P={P}")


def test_a_window_of_everything_is_slot_attn():
    """The whole prefix through either call: the same value but for the rounding of the
    probabilities against another running maximum."""
    dev = require_gpu()
    for heads, S, L in [((4, 2), 1, 1), ((4, 2), 8, 8), ((8, 2), 8, 16)]:
        c = Case(dev, 2, heads, 128, 1000, S, L, seed=8)
        out, lse = c.run()
        out_w, lse_w = c.run(window=1000 + S * L, sinks=0)
        O, _, A = c.ref()
        assert np.all(np.abs((out.float() - out_w.float()).cpu().numpy()) <= 2.0 ** -7 * (A + np.abs(O)) + 2e-3 * A)
        assert (lse - lse_w).abs().max().item() <= 2e-5


def fill_hidden(c, places, value):
    """Give prefix rows `places` of every head keys and values of `value` (a number, or a
    4-bit scale byte)."""
    for name in ("k_cache", "v_cache"):
        c.f[name][:, :, places] = np.nan
    if c.q4:
        for t in c.cache:
            t[:, :, places] = value
    else:
        for name in ("k_cache", "v_cache"):
            c.d[name][:, :, places] = value


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,S,L", [((4, 2), 1, 1), ((2, 1), 3, 5), ((4, 2), 8, 8), ((4, 1), 4, 16)])
def test_values_out_of_sight_never_arrive(heads, S, L, dtype, q4):
    """Rows before the window, beside the sinks and behind the prefix hold NaN and
    infinities; some of them share tiles, or are seen by earlier tokens only."""
    dev = require_gpu()
    T, window, sinks, n = S * L, 70, 3, 301
    for value in ([255, 254] if q4 else [float("nan"), float("inf"), float("-inf")]):
        say(f"hidden {value} {heads} {S}x{L} {dtype} q4={q4}")
        c = Case(dev, 1, heads, 128, 320, S, L, dtype, q4=q4, lens=[n], seed=2, pass_=1, window=window, sinks=sinks)
        first = n - window + 1  # what the first token still sees
        fill_hidden(c, list(range(sinks, first)) + list(range(n, 320)), value)
        check(*c.run(), c.ref(), dtype, f"{value}")
    if T > 1:
        # a key that the first tokens see and the last do not: NaN for those alone
        c = Case(dev, 1, heads, 128, 320, S, L, dtype, q4=q4, lens=[n], seed=2, pass_=1, window=window, sinks=sinks)
        fill_hidden(c, [first + T // 2 - 1], 255 if q4 else float("nan"))
        out, lse = c.run()
        ref = c.ref()
        assert np.isnan(ref[0]).any() and not np.isnan(ref[0]).all()
        check(out, lse, ref, dtype, "seen by the first tokens")
        # a draft token's own value that other slots do not see
        c = Case(dev, 1, heads, 128, 320, S, L, dtype, q4=q4, lens=[n], seed=2, pass_=1, window=window, sinks=sinks)
        for name in ("k_slot", "v_slot"):
            c.f[name][:, :, T - 1] = np.nan
            c.d[name][:, :, T - 1] = float("nan")
        check(*c.run(), c.ref(), dtype, "the last draft token")


@pytest.mark.parametrize("q4", [False, True])
def test_reruns_workspace_contents_and_surroundings(q4):
    """Bit-identical reruns whatever the workspace holds, and nothing written around
    the outputs."""
    dev = require_gpu()
    from paper_2609_19868_amd import _lib

    for heads, S, L in [((4, 2), 1, 1), ((4, 2), 8, 8)]:
        c = Case(dev, 2, heads, 128, 3000, S, L, q4=q4, seed=4, window=2000, sinks=7)
        n = c.d["q"].numel()
        flat = torch.full((n + 512,), 7.0, dtype=torch.bfloat16, device=dev)
        out = flat[256:256 + n].view(c.d["q"].shape)
        rows = n // 128
        lflat = torch.full((rows + 64,), 9.0, device=dev)
        lse = lflat[32:32 + rows].view(c.d["q"].shape[:3])
        first = None
        for fill in (0, 255, 127):
            ws = torch.full((1 << 24,), fill, dtype=torch.uint8, device=dev)
            c.run(out=out, lse=lse, workspace=ws)
            got = (out.clone(), lse.clone())
            assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
            first = got
        assert (flat[:256] == 7).all() and (flat[256 + n:] == 7).all()
        assert (lflat[:32] == 9).all() and (lflat[32 + rows:] == 9).all()
        desc = Z.slot_attn_desc(c.d["q"], c.cache.k if q4 else c.d["k_cache"], c.d["k_slot"], S, L)
        win = _lib.AttnWindow(window=2000, sinks=7)
        need = (_lib.slot_attn_q4_workspace_size if q4 else _lib.slot_attn_window_workspace_size)(desc, win)
        assert need > 0  # the case has splits
        ws = torch.full((need + 256,), 5, dtype=torch.uint8, device=dev)
        c.run(out=out, lse=lse, workspace=ws[:need])
        assert (ws[need:] == 5).all() and torch.equal(out, first[0])


@pytest.mark.parametrize("q4", [False, True])
def test_offsets_past_32_bits(q4):
    """The last rows of a cache whose arrays pass 4 GiB."""
    dev = require_gpu()
    Hkv, C = (4, (1 << 24) + 96) if q4 else (4, (1 << 22) + 96)
    n, window, sinks = C - 1, 50, 2
    say(f"far offsets q4={q4} C={C}")
    g = torch.Generator(device=dev).manual_seed(1)
    small = torch.randn((2, 1, Hkv, 64, 128), generator=g, device=dev).to(torch.bfloat16)
    if q4:
        cache = Z.q4_cache(1, Hkv, C, 128, dev)
        # rows that would give another result if an address lost its upper bits
        cache.k_scale.fill_(130), cache.v_scale.fill_(130), cache.k.fill_(0x5a), cache.v.fill_(0x5a)
        at = torch.tensor([C - 64], dtype=torch.int32, device=dev)
        Z.kv_quantize(small[0], small[1], cache, starts=at)
        k = oracle.q4_dequantize(cache.k[:, :, -64:].cpu().numpy(), cache.k_scale[:, :, -64:].cpu().numpy())
        v = oracle.q4_dequantize(cache.v[:, :, -64:].cpu().numpy(), cache.v_scale[:, :, -64:].cpu().numpy())
        want = [oracle.q4_dequantize(*oracle.q4_quantize(x.float().cpu().numpy())) for x in small]
        assert np.array_equal(k, want[0]) and np.array_equal(v, want[1])
        head = oracle.q4_dequantize(cache.k[:, :, :sinks].cpu().numpy(), cache.k_scale[:, :, :sinks].cpu().numpy())
    else:
        cache = [torch.full((1, Hkv, C, 128), 3.0, dtype=torch.bfloat16, device=dev) for _ in range(2)]
        for t, s in zip(cache, small):
            t[:, :, -64:] = s
        k, v = (s.float().cpu().numpy().astype(np.float64) for s in small)
        head = np.full((1, Hkv, sinks, 128), 3.0)
    lens = torch.tensor([n], dtype=torch.int32, device=dev)
    for S, L, G in [(1, 1, 2), (4, 12, 2)]:
        T = S * L
        q, ks, vs = (torch.randn((1, h, T, 128), generator=g, device=dev).to(torch.bfloat16) for h in (Hkv * G, Hkv, Hkv))
        if q4:
            got = Z.slot_attn_q4(q, cache, ks, vs, S, L, prefix_lens=lens, window=window, sinks=sinks)
        else:
            got = Z.slot_attn(q, cache[0], cache[1], ks, vs, S, L, prefix_lens=lens, window=window, sinks=sinks)
        torch.cuda.synchronize()
        # the same call with the rows in between left out
        f = [t.float().cpu().numpy().astype(np.float64) for t in (q, ks, vs)]
        kk, vv = (np.concatenate([head, x[:, :, :-1]], 2) for x in (k, v))
        ref = oracle.view_attention(f[0], kk, vv, f[1], f[2], sinks + 63, S, L, 128 ** -0.5, 0, window=window, sinks=sinks)
        check(*got, ref, "bf16", f"{S}x{L}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_to_the_code(dtype):
    """Codes and scales equal the oracle's: halves between two magnitudes, subnormal
    and largest values, zeros, blocks with NaN and infinities; odd row counts."""
    dev = require_gpu()
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 3, 129, 128)) * np.exp(3 * rng.standard_normal((2, 3, 129, 1)))
    x[0, 0, 0] = 0
    x[0, 0, 1] = np.resize(np.arange(-32, 33) * 0.25, 128)  # ties of every kind, 7 and 8 among them
    x[0, 0, 2] *= 1e-38
    x[0, 0, 3] = np.resize(np.arange(128) * 2.0 ** -133, 128)  # subnormal in both types
    x[0, 0, 4, 5], x[0, 0, 5, 70], x[0, 0, 6, 100] = np.nan, np.inf, -np.inf
    x[0, 0, 7] = np.resize([3.3e38, -3.3e38, 1e38, 2.2e38, 2.4e38, 5e37], 128)
    x[0, 0, 8] = np.resize([7.0, 6.96875, 1.0, 5.0, 3.5, 2.5], 128)
    x[0, 0, 9] = np.resize([6.96875, 1.0, 5.0, -3.5, -2.5, -0.25], 128)
    host = W.bf16_bits(x.astype(np.float32)) if dtype == "bf16" else x.astype(np.float32)
    f = W.as_f64(host, dtype)
    for D in (128, 64):
        xs = np.ascontiguousarray(host.reshape(2, 3, -1, D))
        N = xs.shape[2] - (D == 64)  # 129 and 257 rows: chunks that end inside
        xd = to_dev(xs, dtype, dev)[:, :, :N].contiguous()
        fs = f.reshape(2, 3, -1, D)[:, :, :N]
        say(f"quantize {dtype} D={D} N={N}")
        cache = Z.kv_quantize(xd, -xd, Z.q4_cache(2, 3, N + 5, D, dev))
        torch.cuda.synchronize()
        for codes, scales, src in ((cache.k, cache.k_scale, fs), (cache.v, cache.v_scale, -fs)):
            qc, qs = oracle.q4_quantize(src)
            want = oracle.q4_dequantize(qc, qs)
            assert np.array_equal(scales[:, :, :N].cpu().numpy(), qs)
            got = oracle.q4_dequantize(codes[:, :, :N].cpu().numpy(), scales[:, :, :N].cpu().numpy())
            assert np.array_equal(got, want, equal_nan=True)  # the sign of a zero may differ
            assert (codes[:, :, N:] == 0).all() and (scales[:, :, N:] == 0).all()
        # the values, in both types, are those of the codes
        for out_dtype in (torch.bfloat16, torch.float32):
            k, v = Z.kv_dequantize(cache, N, out_dtype)
            torch.cuda.synchronize()
            assert np.array_equal(k.double().cpu().numpy(), oracle.q4_dequantize(*oracle.q4_quantize(fs)), equal_nan=True)
            assert np.array_equal(v.double().cpu().numpy(), oracle.q4_dequantize(*oracle.q4_quantize(-fs)), equal_nan=True)


def test_every_code_and_scale_reads_as_its_value():
    dev = require_gpu()
    for D in (64, 128):
        codes = np.resize(np.arange(256, dtype=np.uint8), (1, 1, 256 * 256 // (D // 2), D // 2)).copy()
        rows = codes.shape[2]
        scales = np.broadcast_to((np.arange(rows) * 256 // rows).astype(np.uint8)[None, None, :, None],
                                 (1, 1, rows, D // 32)).copy()
        cache = Z.Q4Cache(*(torch.from_numpy(t).to(dev) for t in (codes, scales, codes, scales)))
        want = oracle.q4_dequantize(codes, scales)
        for dtype in (torch.bfloat16, torch.float32):
            with np.errstate(over="ignore"):
                w = torch.from_numpy(want).to(dtype).double().numpy()  # infinities past the type's range
            k, v = Z.kv_dequantize(cache, dtype=dtype)
            torch.cuda.synchronize()
            assert np.array_equal(k.double().cpu().numpy(), w, equal_nan=True)
            assert np.array_equal(v.double().cpu().numpy(), w, equal_nan=True)


def test_rows_that_are_not_asked_for_stay():
    """Starts and lengths per batch row: rows that do not fit, none, all, out of range."""
    dev = require_gpu()
    B, Hkv, C, D, N = 7, 2, 90, 64, 70
    g = torch.Generator(device=dev).manual_seed(2)
    k, v = (torch.randn((B, Hkv, N, D), generator=g, device=dev) for _ in range(2))
    starts, lens = [0, 20, 21, -1, 89, 5, 90], [70, 70, 70, 3, 1, -4, 99]
    cache = Z.q4_cache(B, Hkv, C, D, dev)
    for t in cache:
        t.fill_(0x33)
    Z.kv_quantize(k, v, cache, torch.tensor(starts, dtype=torch.int32, device=dev),
                  torch.tensor(lens, dtype=torch.int32, device=dev))
    torch.cuda.synchronize()
    for b in range(B):
        n = min(max(lens[b], 0), N)
        if starts[b] < 0 or starts[b] + n > C:
            n = 0
        for codes, scales, x in ((cache.k, cache.k_scale, k), (cache.v, cache.v_scale, v)):
            qc, qs = oracle.q4_quantize(x[b, :, :n].cpu().numpy())
            want_c, want_s = np.full((Hkv, C, D // 2), 0x33, np.uint8), np.full((Hkv, C, D // 32), 0x33, np.uint8)
            want_c[:, starts[b]:starts[b] + n], want_s[:, starts[b]:starts[b] + n] = qc, qs
            assert np.array_equal(codes[b].cpu().numpy(), want_c) and np.array_equal(scales[b].cpu().numpy(), want_s)
    out = tuple(torch.full((B, Hkv, N, D), 5.0, device=dev) for _ in range(2))
    Z.kv_dequantize(cache, N, torch.float32, torch.tensor(lens, dtype=torch.int32, device=dev), out)
    torch.cuda.synchronize()
    for b in range(B):
        n = min(max(lens[b], 0), N)
        assert (out[0][b, :, n:] == 5).all() and (out[1][b, :, n:] == 5).all()
        want = oracle.q4_dequantize(cache.k[b, :, :n].cpu().numpy(), cache.k_scale[b, :, :n].cpu().numpy())
        assert np.array_equal(out[0][b, :, :n].cpu().numpy(), want)
    Z.kv_quantize(k[:, :, :0].contiguous(), v[:, :, :0].contiguous(), cache)  # no rows: nothing to do
    assert Z.kv_dequantize(cache, 0)[0].shape == (B, Hkv, 0, D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,S,L", [(128, 8, 8), (64, 5, 3), (64, 1, 1), (128, 2, 70), (128, 2, 300), (128, 1024, 1), (64, 64, 128)])
def test_append(dtype, D, S, L):
    """The accepted tokens behind each row's prefix, as kv_append puts them there: lists
    that end early or name a slot twice, rows that do not fit."""
    dev = require_gpu()
    rng = np.random.default_rng(S * L + D)
    B, Hkv, C = 6, 3, 40 + S * L // 2
    x = [rng.standard_normal((B, Hkv, S * L, D)).astype(np.float32) for _ in range(2)]
    x = [W.bf16_bits(t) if dtype == "bf16" else t for t in x]
    f = [W.as_f64(t, dtype) for t in x]
    acc = rng.integers(0, 2, (B, S, L)).astype(np.uint8)
    order = np.stack([rng.permutation(S) for _ in range(B)]).astype(np.int32)
    order[1, S // 2:] = -1
    if S > 2:
        order[2, 1] = order[2, 0]
        order[3, 1] = S + 3
    acc[4] = 1
    lens0 = np.array([0, 7, 40, 11, C - 2, -1], np.int32)
    say(f"append {dtype} D={D} {S}x{L}")
    cache = Z.q4_cache(B, Hkv, C, D, dev)
    for t in cache:
        t.fill_(0x42)
    lens = torch.from_numpy(lens0).to(dev)
    Z.kv_append_q4(cache, lens, to_dev(x[0], dtype, dev), to_dev(x[1], dtype, dev), torch.from_numpy(acc).to(dev),
                   torch.from_numpy(order).to(dev))
    torch.cuda.synchronize()
    want = [np.full((B, Hkv, C, n), 0x42, np.uint8) for n in (D // 2, D // 32, D // 2, D // 32)]
    q = [oracle.q4_quantize(t) for t in f]
    want_lens = lens0.copy()
    for b in range(B):
        tokens, done = [], set()
        for s in order[b]:
            if s < 0:
                break
            if s < S and s not in done:
                done.add(s)
                tokens += [s * L + r for r in range(L) if acc[b, s, r]]
        if lens0[b] < 0 or lens0[b] + len(tokens) > C:
            continue
        for i, t in enumerate(tokens):
            for j, part in enumerate((q[0][0], q[0][1], q[1][0], q[1][1])):
                want[j][b, :, lens0[b] + i] = part[b, :, t]
        want_lens[b] += len(tokens)
    assert np.array_equal(lens.cpu().numpy(), want_lens)
    assert (want_lens != lens0).any()
    for got, w in zip(cache, want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_a_run_of_them_together():
    """Prompt into the cache, then draft, verify, append and draft again over the grown
    prefixes, under a window: each stage against the oracle on that stage's inputs."""
    dev = require_gpu()
    B, Hq, Hkv, D, S, L, C = 3, 4, 2, 128, 4, 8, 256
    g = torch.Generator(device=dev).manual_seed(3)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)

    def host(t):
        return t.float().cpu().numpy().astype(np.float64)

    lens = torch.tensor([150, 64, 0], dtype=torch.int32, device=dev)
    cache = Z.kv_quantize(rnd(B, Hkv, 150, D), rnd(B, Hkv, 150, D), Z.q4_cache(B, Hkv, C, D, dev), lens=lens)
    for step in range(3):
        q, ks, vs = rnd(B, Hq, S * L, D), rnd(B, Hkv, S * L, D), rnd(B, Hkv, S * L, D)
        k, v = Z.kv_dequantize(cache)
        for pass_ in (Z.PASS_DIFFUSION, Z.PASS_AR_INFILL):
            say(f"run step {step} pass {pass_}")
            got = Z.slot_attn_q4(q, cache, ks, vs, S, L, pass_=pass_, prefix_lens=lens, window=90, sinks=4)
            again = Z.slot_attn(q, k, v, ks, vs, S, L, pass_=pass_, prefix_lens=lens, window=90, sinks=4)
            torch.cuda.synchronize()
            ref = oracle.view_attention(host(q), host(k), host(v), host(ks), host(vs), lens.tolist(), S, L, D ** -0.5,
                                        pass_, window=90, sinks=4)
            check(*got, ref, "bf16", f"step {step}")
            check(*again, ref, "bf16", f"step {step}, dequantized")
        prob = torch.rand((B, S, L), generator=g, device=dev)
        _, selected, _ = Z.select_slots(prob, rule=Z.SELECT_TOP_K, k=3)
        accepted, _, total = Z.verify_accept(prob, selected, 0.2)
        before = lens.clone()
        Z.kv_append_q4(cache, lens, ks, vs, accepted, selected)
        torch.cuda.synchronize()
        assert torch.equal(lens, before + total)


def test_graph_replays():
    """Quantize, append and both attentions captured once and replayed with new inputs,
    eager work in between; two graphs that share a workspace, one after the other."""
    dev = require_gpu()
    B, Hq, Hkv, D, S, L, C = 2, 4, 2, 128, 1, 1, 2048
    g = torch.Generator(device=dev).manual_seed(4)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)

    prompt = (rnd(B, Hkv, 2000, D), rnd(B, Hkv, 2000, D))
    q, ks, vs = rnd(B, Hq, S * L, D), rnd(B, Hkv, S * L, D), rnd(B, Hkv, S * L, D)
    lens = torch.full((B,), 2000, dtype=torch.int32, device=dev)
    accepted = torch.ones((B, S, L), dtype=torch.uint8, device=dev)
    order = torch.zeros((B, S), dtype=torch.int32, device=dev)
    cache = Z.q4_cache(B, Hkv, C, D, dev)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=dev)
    outs = [torch.empty_like(q) for _ in range(2)]
    lses = [torch.empty((B, Hq, S * L), device=dev) for _ in range(2)]

    def one(i, **kw):
        return Z.slot_attn_q4(q, cache, ks, vs, S, L, prefix_lens=lens, out=outs[i], lse=lses[i], workspace=ws, **kw)

    def first():
        Z.kv_quantize(*prompt, cache)
        one(0)
        Z.kv_append_q4(cache, lens, ks, vs, accepted, order)

    def second():
        one(1, window=700, sinks=4)

    first(), second()
    torch.cuda.synchronize()
    graphs = []
    for fn in (first, second):
        lens.fill_(2000)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fn()
        graphs.append(graph)
    for i in range(4):
        say(f"replay {i}")
        for t in (*prompt, q, ks, vs):
            t.copy_(rnd(*t.shape))
        lens.fill_(1900 + i)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*outs, *lses, lens, *cache)]
        lens.fill_(1900 + i)
        for t in (*outs, *lses):
            t.zero_()
        first(), second()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*outs, *lses, lens, *cache)))


def test_on_another_stream():
    dev = require_gpu()
    c = Case(dev, 1, (4, 2), 128, 1500, 1, 1, q4=True, seed=6)
    want = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = Z.slot_attn_q4(c.d["q"], c.cache, c.d["k_slot"], c.d["v_slot"], 1, 1)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
