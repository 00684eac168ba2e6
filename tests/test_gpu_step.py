"""Steps over request pages on the GPU against the 64-bit oracle: per-head
norms with RoPE and the page write, attention under a window with sinks, 4-bit
pages, and a composed prefill followed by decoding.

Tolerances.  Half a step of a result's type is eps / 2 of its value.  Scores
are fp32 sums of d products: off by at most d 2^-24 of max_j scale sum_i |q_i
k_ji|, which is the relative error it puts on a probability; exp2 and its
argument add 2^-19; splitting a probability into two bf16 parts 2^-17, rounding
it to fp16 2^-11.  Sums over n keys add n 2^-24.  An output is a quotient of two
such sums: twice that, of sum_j p_j |v_j|.  fp32 models compute in fp64 and
round once."""
from types import SimpleNamespace as NS

import numpy as np
import pytest
import torch

import paper_2609_32999_amd as P
import workloads
from oracle import rope as R
from oracle import step as O
from oracle.numerics import round_bf16
from paper_2609_32999_amd import staging
from paper_2609_32999_amd.session import Session

pytestmark = [pytest.mark.gpu]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
FP16 = 2.0 ** -11     # probabilities rounded to fp16 (the kernel for many rows)


def part_of(step):
    return FP16 if step.attn_item_rows == 256 else 2.0 ** -17


def shape(hq=8, hkv=2, d=128, page=16, kv="bf16", max_position=8192):
    return workloads.ModelShape(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page,
                                kv_dtype=kv, act_dtype=kv, max_position=max_position)


def rand(gen, *s, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(s, generator=gen, dtype=torch.float32) * scale).to(dtype).cuda()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def f64(t):
    return t.double().cpu().numpy()


def batch(lens_rows, page, seed=0, spare=3):
    """Requests of (kv_len, positions or row count, row_lo or None) over
    shuffled pages; returns them and the arena's page count."""
    n = sum(-(-l // page) for l, *_ in lens_rows) + spare
    ids = np.random.default_rng(seed).permutation(n).tolist()
    reqs = []
    for l, rows, *lo in lens_rows:
        k = -(-l // page)
        pos = None if isinstance(rows, int) else list(rows)
        reqs.append(NS(kv_len=l, n_rows=rows if pos is None else len(pos), positions=pos,
                       row_lo=lo[0] if lo else None, block_table=ids[:k]))
        ids = ids[k:]
    return reqs, n


def row_list(reqs):
    """(request, position, lo) of every row."""
    out = []
    for i, r in enumerate(reqs):
        pos = r.positions or range(r.kv_len - r.n_rows, r.kv_len)
        lo = r.row_lo or [0] * r.n_rows
        out += [(i, p, l) for p, l in zip(pos, lo)]
    return out


def request_kv(pages, r, n):
    """[n][H_kv][..] of a request from its pages."""
    t = pages[torch.tensor(r.block_table, device=pages.device, dtype=torch.long)]
    return t.transpose(1, 2).reshape(-1, t.shape[1], *t.shape[3:])[:n]


def check_attn(reqs, q, out, lse, kv, d, n_keys, window=0, n_sinks=0, f32=False, part=2.0 ** -17):
    """kv(i): fp64 K, V of request i, [kv_len][H_kv][d]."""
    rows, at = row_list(reqs), 0
    half = torch.finfo(out.dtype).eps / 2
    for i, r in enumerate(reqs):
        mine = [x for x in rows if x[0] == i]
        if not mine:
            continue
        K, V = kv(i)
        sl = slice(at, at + len(mine))
        ref, rl, mag, top = O.step_attention(f64(q[sl]), [x[1] for x in mine],
                                             [x[2] for x in mine], K, V, window, n_sinks)
        at += len(mine)
        if f32:
            rel = np.full_like(top, 2.0 ** -40)
        else:
            rel = d * 2.0 ** -24 * top + 2.0 ** -19 + n_keys * 2.0 ** -24
        got, gl = f64(out[sl]), f64(lse[sl])
        # partial rows of cut key ranges are kept in fp32
        tol = half * np.abs(ref) * (1 + 2 * rel[..., None]) + \
            (2 * (rel + (0 if f32 else part))[..., None] + 2.0 ** -22) * mag
        if part == FP16:            # values below fp16's normal range: half its step
            tol += 2.0 ** -25
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        bad = ~(np.abs(got - ref) <= tol) & ~np.isnan(ref)
        assert not bad.any(), (i, np.argwhere(bad)[:5], np.abs(got - ref)[bad][:5], tol[bad][:5])
        none = np.isneginf(rl)
        assert np.array_equal(np.isneginf(gl), none) and not got[none].any()
        ok = np.isfinite(rl)
        assert np.array_equal(np.isnan(gl), np.isnan(rl))
        assert (np.abs(gl[ok] - rl[ok]) <= (rel + 2.0 ** -22 * (1 + np.abs(rl)))[ok]).all()


def run_attn(sh, reqs, n_pages, seed, poison=None, **opt):
    """Random pages (every slot not a position of a request NaN) through a step."""
    g = gen(seed)
    dt = DT[sh.kv_dtype]
    sess = Session(sh, 1, n_pages)
    sess.req_k.fill_(float("nan"))
    sess.req_v.fill_(float("nan"))
    for r in reqs:
        for t in (sess.req_k[0], sess.req_v[0]):
            for j, pg in enumerate(r.block_table):
                n = min(sh.page_size, r.kv_len - j * sh.page_size)
                t[pg, :, :n] = rand(g, sh.n_kv_heads, n, sh.head_dim, dtype=dt)
    if poison:
        poison(sess)
    step = sess.step(reqs, **opt)
    q = rand(g, step.num_rows, sh.n_q_heads, sh.head_dim, dtype=dt, scale=1.5)
    out = torch.full_like(q, float("nan"))
    lse = torch.full((step.num_rows, sh.n_q_heads), float("nan"), device="cuda")
    sess.step_attn(step, q, out, lse)
    torch.cuda.synchronize()
    return sess, step, q, out, lse


def pages_kv(sess, reqs):
    return lambda i: (f64(request_kv(sess.req_k[0], reqs[i], reqs[i].kv_len)),
                      f64(request_kv(sess.req_v[0], reqs[i], reqs[i].kv_len)))


# -------------------------------------------------------------- attention
CASES = {
    # name: (shape, requests, options)
    "one_key": (dict(), [(1, 1)], dict()),
    "one_token": (dict(), [(77, 1)], dict()),
    "decode": (dict(), [(33, 1), (1, 1), (160, 1), (16, 1), (300, 1)], dict()),
    "rows": (dict(), [(95, 40), (17, 17), (5, 2)], dict()),
    "window": (dict(), [(700, 1), (40, 1), (333, 9)], dict(window=64, n_sinks=4)),
    "window_one": (dict(), [(70, 3)], dict(window=1)),
    "window_sinks_meet": (dict(), [(90, 60)], dict(window=30, n_sinks=33)),
    "sinks_wide": (dict(), [(500, 5)], dict(window=16, n_sinks=200)),
    "cut": (dict(), [(1000, 1), (64, 1), (31, 2)], dict(split_tiles=1)),
    "cut_window": (dict(), [(999, 2), (450, 1)], dict(split_tiles=3, window=200, n_sinks=70)),
    "cut_odd": (dict(), [(2001, 1)], dict(split_tiles=7)),
    "cut_pairs": (dict(), [(64, 3), (50, 1), (20, 1)], dict(split_tiles=1)),
    "mha": (dict(hq=4, hkv=4), [(60, 21), (130, 1)], dict(window=50, n_sinks=1)),
    "g3": (dict(hq=6, hkv=2), [(61, 7), (130, 1)], dict()),
    "g8": (dict(hq=16, hkv=2), [(45, 5), (200, 1)], dict(split_tiles=2)),
    "g16": (dict(hq=32, hkv=2), [(45, 3)], dict()),
    "g20": (dict(hq=20, hkv=1), [(45, 3), (70, 1)], dict(window=20)),
    "page32": (dict(page=32), [(95, 4), (31, 1), (33, 1)], dict(window=40, n_sinks=2)),
    "page64": (dict(page=64), [(190, 4), (64, 1)], dict()),
    # enough rows for the kernel for many
    "many": (dict(), [(300, 300), (700, 150)], dict()),
    "many_window": (dict(), [(500, 400), (64, 64)], dict(window=70, n_sinks=5)),
    "many_window_one": (dict(), [(140, 140)], dict(window=1, n_sinks=1)),
    "many_cut": (dict(), [(900, 90)], dict(split_tiles=3)),
    "many_cut_window": (dict(), [(900, 300)], dict(split_tiles=2, window=100, n_sinks=40)),
    "many_and_few": (dict(), [(900, 1), (700, 600), (77, 2), (90, 16)], dict()),
    "many_mha": (dict(hq=2, hkv=2), [(530, 530)], dict(window=300)),
    "many_g5": (dict(hq=10, hkv=2), [(260, 130), (64, 20)], dict()),
    "many_g20": (dict(hq=20, hkv=1), [(99, 50)], dict()),
    "many_g64": (dict(hq=64, hkv=1), [(99, 9)], dict(window=33, n_sinks=2)),
    "many_page64": (dict(page=64), [(400, 200)], dict()),
    "many_spread": (dict(), [(900, sorted(range(3, 900, 7)))], dict(window=128, n_sinks=8)),
    "many_lo": (dict(), [(600, list(range(200, 330)), [200 + 50 * (i // 50) for i in range(130)])],
                dict()),
    "many_nothing": (dict(), [(600, [-1] * 70 + list(range(100, 200)),
                               [0] * 70 + [100 + i + (i % 3 == 0) for i in range(100)])], dict()),
    "spread": (dict(), [(200, [0, 3, 77, 78, 150, 199]), (90, [10, 40])], dict()),
    "lo": (dict(), [(200, [20, 40, 120, 199], [0, 33, 100, 64])], dict(window=30, n_sinks=6)),
    "nothing": (dict(), [(50, [-1, 10, -1, 20, 49], [0, 11, 0, 0, 50]), (0, [-1, -1])], dict()),
    "nothing_cut": (dict(), [(300, [-1, 200, 299], [0, 201, 250])], dict(split_tiles=1)),
    "f32": (dict(hq=4, hkv=4, d=64, kv="f32"), [(272, [3, 99, 100, 271]), (9, 1)],
            dict(window=60, n_sinks=3)),
    "f32_page8": (dict(hq=6, hkv=2, kv="f32", page=8), [(50, 20), (1, 1)], dict()),
    "f32_256": (dict(hq=4, hkv=2, d=256, kv="f32"), [(70, 9)], dict(split_tiles=1)),
    "f32_pairs": (dict(hq=4, hkv=2, kv="f32"), [(64, 3), (50, 1), (20, 1)],
                  dict(split_tiles=1)),
    "f32_lo": (dict(hq=4, hkv=1, d=64, kv="f32"), [(90, [-1, 20, 89], [0, 21, 40])],
               dict(split_tiles=1, window=33, n_sinks=2)),
}


@pytest.mark.parametrize("name,kernel", [(n, 0) for n in CASES] +
                         [(n, 2) for n in CASES if n[:3] != "f32"] +
                         [(n, 1) for n in CASES if n[:4] == "many"])
def test_attention(name, kernel):
    sh, lens, opt = CASES[name]
    sh, opt = shape(**sh), dict(opt, attn_kernel=kernel)
    reqs, n = batch(lens, sh.page_size, seed=len(name))
    sess, step, q, out, lse = run_attn(sh, reqs, n, len(name) * 7, **opt)
    assert step.num_attn_splits > 0 or "split_tiles" not in opt
    check_attn(reqs, q, out, lse, pages_kv(sess, reqs), sh.head_dim,
               max(r.kv_len for r in reqs), opt.get("window", 0), opt.get("n_sinks", 0),
               f32=sh.kv_dtype == "f32", part=part_of(step))


@pytest.mark.parametrize("kv,d,kernel", [("bf16", 128, 1), ("bf16", 128, 2), ("f32", 64, 0)])
@pytest.mark.parametrize("split", [-1, 1])
def test_unseen_values_stay_out(kv, d, kernel, split):
    """Infinities and NaN at keys a row does not see, seen by other rows of
    the same item or by none, and values that a row sees."""
    sh = shape(hq=4, hkv=1, d=d, kv=kv)
    # rows at 40, 41, 70: the first two share key tiles with keys past them
    reqs, n = batch([(96, [40, 41, 70, 95], [0, 0, 10, 64])], 16)
    t = reqs[0].block_table

    def poison(s):
        for key, x in ((41, float("inf")), (70, float("nan")), (3, float("-inf"))):
            s.req_v[0, t[key // 16], 0, key % 16, 5] = x
        s.req_k[0, t[60 // 16], 0, 60 % 16, 1] = float("nan")
        s.req_k[0, t[50 // 16], 0, 50 % 16] = float("inf")

    sess, step, q, out, lse = run_attn(sh, reqs, n, 5, poison=poison, split_tiles=split,
                                       window=25, n_sinks=2, attn_kernel=kernel)
    # row 40: keys 0, 1, 16 .. 40: nothing bad.  Row 41 sees the inf at dim 5.
    assert torch.isfinite(out[0]).all() and torch.isfinite(lse[0]).all()
    assert torch.isinf(out[1, :, 5]).all()
    assert torch.isfinite(out[1, :, :5]).all() and torch.isfinite(lse[1]).all()
    assert torch.isnan(out[2]).any() and torch.isnan(lse[2]).any()       # its own keys
    # row 95 sees 64, 65, 71 .. 95
    assert torch.isfinite(out[3]).all() and torch.isfinite(lse[3]).all()
    check_attn([NS(kv_len=96, n_rows=1, positions=[40], row_lo=[0], block_table=t)], q[:1],
               out[:1], lse[:1],
               lambda i: (np.nan_to_num(f64(request_kv(sess.req_k[0], reqs[0], 96)), posinf=0),
                          np.nan_to_num(f64(request_kv(sess.req_v[0], reqs[0], 96)), posinf=0,
                                        neginf=0)), d, 96, 25, 2, f32=kv == "f32",
               part=part_of(step))


@pytest.mark.parametrize("kernel", [1, 2])
def test_equal_and_extreme_scores(kernel):
    """Equal keys give the mean of the values; one huge score takes all."""
    sh = shape(hq=4, hkv=1)
    reqs, n = batch([(130, 1)], 16)
    t = reqs[0].block_table

    def flat(s):
        for pg in t:
            s.req_k[0, pg] = 0.5

    sess, step, q, out, lse = run_attn(sh, reqs, n, 3, poison=flat, attn_kernel=kernel)
    K, V = pages_kv(sess, reqs)(0)
    check_attn(reqs, q, out, lse, pages_kv(sess, reqs), 128, 130, part=part_of(step))
    assert np.abs(f64(out[0, 0]) - V[:, 0].mean(0)).max() < 2.0 ** -8

    def spike(s):
        s.req_k[0, t[4], 0, 2] = 100.0

    sess, step, q, out, lse = run_attn(sh, reqs, n, 3, poison=spike, split_tiles=1,
                                       attn_kernel=kernel)
    check_attn(reqs, q, out, lse, pages_kv(sess, reqs), 128, 130, part=part_of(step))


@pytest.mark.parametrize("kernel", [1, 2])
def test_offsets_past_32_bits(kernel):
    """Pages whose byte offsets pass 2^32 (and whose scale offsets pass 2^28)."""
    sh = shape(hq=8, hkv=8)
    n = (1 << 32) // (8 * 16 * 128 * 2) + 40
    reqs = [NS(kv_len=100, n_rows=2, positions=None, row_lo=None,
               block_table=[n - 1 - 3 * i for i in range(7)])]
    sess = Session(sh, 1, n)
    g = gen(9)
    for pg in reqs[0].block_table:
        sess.req_k[0, pg] = rand(g, 8, 16, 128)
        sess.req_v[0, pg] = rand(g, 8, 16, 128)
    step = sess.step(reqs, attn_kernel=kernel)
    q = rand(g, 2, 8, 128)
    out, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
    sess.step_attn(step, q, out, lse)
    torch.cuda.synchronize()
    check_attn(reqs, q, out, lse, pages_kv(sess, reqs), 128, 100, part=part_of(step))
    k, v = rand(g, 2, 8, 128), rand(g, 2, 8, 128)
    sess.step_append(step, q, k, v, torch.empty_like(q))
    torch.cuda.synchronize()
    assert torch.equal(sess.req_v[0, n - 19, :, 2], v[0])


# ------------------------------------------------------------------ append
def append_case(kv, hq, hkv, d, page, weights, four_bit=False, seed=1):
    sh = shape(hq, hkv, d, page, kv)
    reqs, n = batch([(50, [0, 7, 8, 49]), (page * 3, 1), (90, [-1, 5, 89, -1]), (300, 33)], page,
                    seed)
    g = gen(seed)
    dt = DT[kv]
    sess = Session(sh, 1, n, four_bit=four_bit)
    step = sess.step(reqs, four_bit=four_bit)
    T = step.num_rows
    qkv = rand(g, T, (hq + 2 * hkv) * d + 16, dtype=dt, scale=3.0)   # rows further apart
    q, k, v = (x.unflatten(1, (-1, d)) for x in
               qkv[:, :(hq + 2 * hkv) * d].split([hq * d, hkv * d, hkv * d], 1))
    wq, wk = (rand(g, d, dtype=dt), rand(g, d, dtype=dt)) if weights else (None, None)
    return sess, step, reqs, q, k, v, wq, wk


def check_rotated(got, x, pos, half):
    """got [..][d] against RoPE of fp64 x at pos; cos, sin and the products are
    fp32: 2^-22 of each product."""
    d = x.shape[-1]
    cs, sn = (t.reshape(len(pos), 1, -1) for t in R.cos_sin_fp64(pos, d, 500000.0))
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    ref = np.concatenate([lo * cs - hi * sn, hi * cs + lo * sn], -1)
    mag = np.concatenate([np.abs(lo * cs) + np.abs(hi * sn), np.abs(hi * cs) + np.abs(lo * sn)], -1)
    # the norm: a sum of d squares, a root and two products, each within 2^-23
    tol = half * np.abs(ref) * (1 + 1e-4) + ((d + 8) * 2.0 ** -24 + 2.0 ** -20) * mag
    assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()


@pytest.mark.parametrize("kv,hq,hkv,d,page,weights,norm", [
    ("bf16", 8, 2, 128, 16, True, True), ("bf16", 5, 5, 128, 64, False, True),
    ("bf16", 40, 8, 128, 32, True, True), ("bf16", 4, 1, 128, 16, False, False),
    ("f32", 4, 4, 64, 8, True, True), ("f32", 6, 2, 128, 16, False, False),
    ("f32", 3, 1, 256, 64, True, True)])
def test_append(kv, hq, hkv, d, page, weights, norm):
    sess, step, reqs, q, k, v, wq, wk = append_case(kv, hq, hkv, d, page, weights)
    T = step.num_rows
    for t in (sess.req_k, sess.req_v):
        t.fill_(7.0)
    q_out = torch.full((T, hq, d), 9.0, dtype=q.dtype, device="cuda")
    k_pre = torch.full((T, hkv, d), 9.0, dtype=q.dtype, device="cuda")
    sess.step_append(step, q, k, v, q_out, k_pre, wq, wk, EPS if norm else None)
    torch.cuda.synchronize()
    rows = row_list(reqs)
    live = [t for t in range(T) if rows[t][1] >= 0]
    pos = [rows[t][1] for t in live]
    half = torch.finfo(q.dtype).eps / 2
    qn, kn = f64(q[live]), f64(k[live])
    if norm:
        qn = O.rms_norm(qn, None if wq is None else f64(wq), EPS)
        kn = O.rms_norm(kn, None if wk is None else f64(wk), EPS)
    check_rotated(f64(q_out[live]), qn, pos, half)
    kp = f64(k_pre[live])
    assert (np.abs(kp - kn) <= (half + (d + 8) * 2.0 ** -24) * np.abs(kn)).all()
    # K is the rotation of the very k_pre, with the bits compose would write
    rot = R.rope_fp32(kp.astype(np.float32), pos, 500000.0)
    want_k, want_v = torch.full_like(sess.req_k[0], 7.0), torch.full_like(sess.req_v[0], 7.0)
    for n, t in enumerate(live):
        i, p, _ = rows[t]
        x = rot[n] if kv == "f32" else round_bf16(rot[n])
        want_k[reqs[i].block_table[p // page], :, p % page] = torch.from_numpy(
            np.asarray(x, dtype=np.float32)).to(q.dtype).cuda()
        want_v[reqs[i].block_table[p // page], :, p % page] = v[t]
    assert torch.equal(sess.req_k[0], want_k) and torch.equal(sess.req_v[0], want_v)
    # rows without a token left everything as it was
    pad = [t for t in range(T) if rows[t][1] < 0]
    assert len(pad) == 2 and (q_out[pad] == 9).all() and (k_pre[pad] == 9).all()
    # in place, packed
    q2, k2 = q.contiguous(), k.contiguous()
    sess.step_append(step, q2, k2, v, q2, k2, wq, wk, EPS if norm else None)
    torch.cuda.synchronize()
    assert torch.equal(q2[live], q_out[live]) and torch.equal(k2[live], k_pre[live])
    assert torch.equal(q2[pad], q[pad]) and torch.equal(sess.req_k[0], want_k)


def test_append_many_rows_equal_few():
    """Rows appended all at once and 50 at a time: the same bits."""
    sh = shape(32, 8, max_position=65536)
    g = gen(4)
    T = 700
    q, k, v, wq, wk = (rand(g, T, 32, 128), rand(g, T, 8, 128), rand(g, T, 8, 128), rand(g, 128),
                       rand(g, 128))
    reqs, n = batch([(60000, sorted(np.random.default_rng(0).permutation(60000)[:T].tolist()))], 16)
    sess = Session(sh, 1, n)
    a, ka = torch.empty_like(q), torch.empty_like(k)
    sess.req_k.zero_(), sess.req_v.zero_()
    sess.step_append(sess.step(reqs), q, k, v, a, ka, wq, wk, EPS)
    torch.cuda.synchronize()
    wk_k, wk_v = sess.req_k.clone(), sess.req_v.clone()
    sess.req_k.zero_(), sess.req_v.zero_()
    b, kb = torch.empty_like(q), torch.empty_like(k)
    for i in range(0, T, 50):
        part = [NS(kv_len=60000, n_rows=50, positions=reqs[0].positions[i:i + 50], row_lo=None,
                   block_table=reqs[0].block_table)]
        sess.step_append(sess.step(part), q[i:i + 50], k[i:i + 50], v[i:i + 50], b[i:i + 50],
                         kb[i:i + 50], wq, wk, EPS)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(ka, kb)
    assert torch.equal(sess.req_k, wk_k) and torch.equal(sess.req_v, wk_v)


def test_append_matches_compose():
    """A unit whose k_pre is retained and composed again holds append's bits."""
    sh = shape(32, 8)
    page, n = 16, 40
    reqs, pages = batch([(n, n)], page)
    g = gen(2)
    sess = Session(sh, 4, pages)
    q, k, v = rand(g, n, 32, 128), rand(g, n, 8, 128), rand(g, n, 8, 128)
    q_out, k_pre = torch.empty_like(q), torch.empty_like(k)
    sess.step_append(sess.step(reqs), q, k, v, q_out, k_pre, None, rand(g, 128), EPS)
    unit = NS(unit_id=1, position=0, n_tokens=n, residency=0, n_recompute=0, retain=1,
              pool_pages=np.arange(3, dtype=np.int32))
    req = NS(prompt_len=n, units=[unit], text_segs=[], block_table=reqs[0].block_table)
    sess.retain(sess.plan([req]), k_pre, v)
    want_k = request_kv(sess.req_k[0], reqs[0], n).clone()
    sess.req_k.zero_()
    unit.residency, unit.retain = 1, 0
    sess.compose(sess.plan([req]))
    torch.cuda.synchronize()
    assert torch.equal(request_kv(sess.req_k[0], reqs[0], n), want_k)


# ------------------------------------------------------------- 4-bit pages
def four_bit_kv(sess, reqs):
    return lambda i: tuple(
        O.e2m1_decode(request_kv(c[0], reqs[i], reqs[i].kv_len).cpu().numpy(),
                      request_kv(sess.req4_scale[0][:, w], reqs[i], reqs[i].kv_len).cpu().numpy())
        for w, c in enumerate((sess.req4_k, sess.req4_v)))


@pytest.mark.parametrize("page,hkv", [(16, 2), (32, 3), (64, 1)])
def test_pack_and_unpack(page, hkv):
    sh = shape(4 * hkv, hkv, page=page)
    reqs, n = batch([(100, 1), (page, 1), (1, 1), (page * 2 + 5, 1)], page)
    # a page two requests share, one of them only part of it
    reqs.append(NS(kv_len=page + 3, n_rows=1, positions=None, row_lo=None,
                   block_table=reqs[0].block_table[:2]))
    sess = Session(sh, 1, n, four_bit=True)
    g = gen(page)
    sess.req_k[0] = rand(g, n, hkv, page, 128, scale=2.0)
    # every exponent, halfway points, zeros, subnormals
    sess.req_v[0] = (torch.randint(-15, 16, (n, hkv, page, 128), generator=g) *
                     torch.exp2(torch.randint(-136, 126, (n, hkv, page, 1), generator=g).float())
                     ).to(torch.bfloat16).cuda()
    t = reqs[0].block_table
    sess.req_v[0, t[0], 0, 0, :64] = 0
    sess.req_v[0, t[0], 0, 1, 3] = float("nan")
    sess.req_v[0, t[0], 0, 2, 100] = float("-inf")
    for c in (sess.req4_k, sess.req4_v, sess.req4_scale):
        c.fill_(0x55)
    step = sess.step(reqs, four_bit=True)
    sess.pack_step(step)
    torch.cuda.synchronize()
    live = torch.zeros(n, page, dtype=torch.bool, device="cuda")
    for r in reqs:
        for j, pg in enumerate(r.block_table):
            live[pg, :min(page, r.kv_len - j * page)] = True
    for w, (src, codes) in enumerate(((sess.req_k, sess.req4_k), (sess.req_v, sess.req4_v))):
        ec, es = O.e2m1_encode(f64(src[0]))
        bad = es == 255                       # the codes of a NaN block are free
        got_c, got_s = codes[0].cpu().numpy(), sess.req4_scale[0][:, w].cpu().numpy()
        m = live[:, None, :, None].cpu().numpy()
        assert np.array_equal(got_s[np.broadcast_to(m, got_s.shape)],
                              es[np.broadcast_to(m, es.shape)])
        mc = np.broadcast_to(m, got_c.shape) & ~np.repeat(bad, 16, -1)
        assert np.array_equal(got_c[mc], ec[mc])
        assert (got_c[~np.broadcast_to(m, got_c.shape)] == 0x55).all()
    src_k, src_v = sess.req_k.clone(), sess.req_v.clone()
    sess.req_k.fill_(3.0), sess.req_v.fill_(3.0)
    sess.unpack_step(step)
    torch.cuda.synchronize()
    for w, (src, back, codes) in enumerate(((src_k, sess.req_k, sess.req4_k),
                                            (src_v, sess.req_v, sess.req4_v))):
        want = O.e2m1_decode(codes[0].cpu().numpy(), sess.req4_scale[0][:, w].cpu().numpy())
        want = np.where(live[:, None, :, None].cpu().numpy(), want, 3.0)
        np.testing.assert_array_equal(f64(back[0]), want.astype(np.float32))


def test_unpack_any_codes_and_scales():
    """Pages that others wrote: all 16 codes under all 256 scale bytes."""
    sh = shape(2, 2)
    reqs, n = batch([(64, 1)], 16)
    sess = Session(sh, 1, n, four_bit=True)
    g = gen(5)
    for c in (sess.req4_k, sess.req4_v):
        c.copy_(torch.randint(0, 256, c.shape, generator=g, dtype=torch.uint8))
    # 256 scales a page, half of them K's: every byte of either in two pages
    for i, pg in enumerate(reqs[0].block_table):
        sess.req4_scale[0, pg] = (torch.arange(256).roll(128 * i).to(torch.uint8)
                                  .reshape(sess.req4_scale.shape[2:]).cuda())
    sess.unpack_step(sess.step(reqs, four_bit=True))
    torch.cuda.synchronize()
    t = torch.tensor(reqs[0].block_table)
    for w, (back, codes) in enumerate(((sess.req_k, sess.req4_k), (sess.req_v, sess.req4_v))):
        want = O.e2m1_decode(codes[0][t].cpu().numpy(), sess.req4_scale[0][t, w].cpu().numpy())
        with np.errstate(over="ignore"):
            want = want.astype(np.float32)   # past fp32: infinite in bf16 too
        np.testing.assert_array_equal(f64(back[0][t]), want)


def test_append_to_four_bit_pages():
    sess, step, reqs, q, k, v, wq, wk = append_case("bf16", 8, 2, 128, 16, True, four_bit=True)
    T = step.num_rows
    for c in (sess.req4_k, sess.req4_v, sess.req4_scale):
        c.fill_(0x55)
    q_out = torch.empty(T, 8, 128, dtype=q.dtype, device="cuda")
    k_pre = torch.empty(T, 2, 128, dtype=q.dtype, device="cuda")
    sess.step_append(step, q, k, v, q_out, k_pre, wq, wk, EPS)
    # bf16 pages: the same queries and keys before RoPE
    step2 = sess.step(reqs)
    q2, k2 = torch.empty_like(q_out), torch.empty_like(k_pre)
    sess.step_append(step2, q, k, v, q2, k2, wq, wk, EPS)
    torch.cuda.synchronize()
    rows = row_list(reqs)
    live = [t for t in range(T) if rows[t][1] >= 0]
    assert torch.equal(q2[live], q_out[live]) and torch.equal(k2[live], k_pre[live])
    rot = R.rope_fp32(f64(k_pre[live]).astype(np.float32), [rows[t][1] for t in live], 500000.0)
    kc, ks = O.e2m1_encode(rot)
    vc, vs = O.e2m1_encode(f64(v[live]))
    want = [torch.full_like(x[0], 0x55) for x in (sess.req4_k, sess.req4_v, sess.req4_scale)]
    for n, t in enumerate(live):
        i, p, _ = rows[t]
        at = reqs[i].block_table[p // 16]
        want[0][at, :, p % 16] = torch.from_numpy(kc[n]).cuda()
        want[1][at, :, p % 16] = torch.from_numpy(vc[n]).cuda()
        want[2][at, 0, :, p % 16] = torch.from_numpy(ks[n]).cuda()
        want[2][at, 1, :, p % 16] = torch.from_numpy(vs[n]).cuda()
    assert torch.equal(sess.req4_k[0], want[0]) and torch.equal(sess.req4_v[0], want[1])
    assert torch.equal(sess.req4_scale[0], want[2])


FOUR_BIT = ["many", "many_window", "many_cut_window", "many_and_few", "many_g5", "many_page64",
            "many_nothing", "one_key", "decode", "rows", "window", "cut", "cut_window", "g3", "g8", "g20", "page32",
            "page64", "lo", "nothing", "nothing_cut"]


@pytest.mark.parametrize("name,kernel", [(n, 0) for n in FOUR_BIT] +
                         [(n, 2) for n in FOUR_BIT])
def test_four_bit_attention(name, kernel):
    sh, lens, opt = CASES[name]
    sh, opt = shape(**sh), dict(opt, attn_kernel=kernel)
    reqs, n = batch(lens, sh.page_size, seed=len(name))
    g = gen(len(name))
    sess = Session(sh, 1, n, four_bit=True)
    sess.req_k[0] = rand(g, n, sh.n_kv_heads, sh.page_size, 128)
    sess.req_v[0] = rand(g, n, sh.n_kv_heads, sh.page_size, 128)
    sess.req4_scale.fill_(255)                # slots without a token read as NaN
    sess.req4_k.fill_(0x77), sess.req4_v.fill_(0x77)
    step = sess.step(reqs, four_bit=True, **opt)
    sess.pack_step(step)
    q = rand(g, step.num_rows, sh.n_q_heads, 128, scale=1.5)
    out = torch.full_like(q, float("nan"))
    lse = torch.full((step.num_rows, sh.n_q_heads), float("nan"), device="cuda")
    sess.step_attn(step, q, out, lse)
    torch.cuda.synchronize()
    check_attn(reqs, q, out, lse, four_bit_kv(sess, reqs), 128, max(r.kv_len for r in reqs),
               opt.get("window", 0), opt.get("n_sinks", 0), part=part_of(step))


@pytest.mark.parametrize("kernel", [1, 2])
def test_four_bit_nan_block_reaches_only_its_rows(kernel):
    sh = shape(4, 1)
    reqs, n = batch([(80, [39, 60, 79])], 16)
    sess = Session(sh, 1, n, four_bit=True)
    g = gen(6)
    sess.req_k[0], sess.req_v[0] = rand(g, n, 1, 16, 128), rand(g, n, 1, 16, 128)
    sess.req_v[0, reqs[0].block_table[2], 0, 40 % 16, 70] = float("inf")    # key 40, dims 64 .. 95
    step = sess.step(reqs, four_bit=True, attn_kernel=kernel)
    sess.pack_step(step)
    q = rand(g, 3, 4, 128)
    out = torch.empty_like(q)
    sess.step_attn(step, q, out)
    torch.cuda.synchronize()
    assert torch.isfinite(out[0]).all()
    assert torch.isnan(out[1:, :, 64:96]).all()
    assert torch.isfinite(out[1:, :, :64]).all() and torch.isfinite(out[1:, :, 96:]).all()


def copied(sess, reqs, q, **opt):
    """The requests as often as the kernel for many rows needs for more work
    items than a launch with a workgroup on each unit holds: outputs, [copies]
    [rows][heads][d] and [copies][rows][heads]."""
    opt = {"split_tiles": -1, **opt}   # automatic ranges go by the whole batch
    one = sess.step(reqs, attn_kernel=2, **opt)
    k = 256 // one.num_attn_items + 1
    step = sess.step(list(reqs) * k, attn_kernel=2, **opt)
    assert step.num_attn_items > 256 and step.attn_item_rows == 256
    qk = q.repeat(k, 1, 1)
    out = torch.full_like(qk, float("nan"))
    lse = torch.full(qk.shape[:2], float("nan"), device="cuda")
    sess.step_attn(step, qk, out, lse)
    torch.cuda.synchronize()
    return out.unflatten(0, (k, -1)), lse.unflatten(0, (k, -1))


def same_bits(t):
    """Every copy's bits are the first's."""
    w = t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
    return bool((w == w[:1]).all())


@pytest.mark.parametrize("four_bit", [False, True])
@pytest.mark.parametrize("name", ["one_key", "decode", "window_one", "window_sinks_meet", "lo",
                                  "nothing", "nothing_cut", "cut_window", "g20", "page64", "many",
                                  "many_window", "many_cut_window", "many_mha", "many_g5",
                                  "many_spread", "many_lo", "many_nothing"])
def test_full_launch(name, four_bit):
    """More work items than units: the other form of the kernel for many rows."""
    sh, lens, opt = CASES[name]
    sh = shape(**sh)
    reqs, n = batch(lens, sh.page_size, seed=len(name))
    sess, _, q, _, _ = run_attn(sh, reqs, n, len(name), **opt)
    kv = pages_kv(sess, reqs)
    if four_bit:
        bf = sess
        sess = Session(sh, 1, n, four_bit=True)
        sess.req_k.copy_(bf.req_k), sess.req_v.copy_(bf.req_v)
        sess.req4_scale.fill_(255)
        sess.req4_k.fill_(0x77), sess.req4_v.fill_(0x77)
        sess.pack_step(sess.step(reqs, four_bit=True))
        kv = four_bit_kv(sess, reqs)
    out, lse = copied(sess, reqs, q, four_bit=four_bit, **opt)
    check_attn(reqs, q, out[0], lse[0], kv, 128, max(r.kv_len for r in reqs),
               opt.get("window", 0), opt.get("n_sinks", 0), part=FP16)
    assert same_bits(out) and same_bits(lse)


@pytest.mark.parametrize("split", [-1, 1])
def test_unseen_values_stay_out_of_a_full_launch(split):
    sh = shape(hq=4, hkv=1)
    reqs, n = batch([(96, [40, 41, 70, 95], [0, 0, 10, 64]), (300, 140)], 16)
    t = reqs[0].block_table

    def poison(s):
        for key, x in ((41, float("inf")), (70, float("nan")), (3, float("-inf"))):
            s.req_v[0, t[key // 16], 0, key % 16, 5] = x
        s.req_k[0, t[60 // 16], 0, 60 % 16, 1] = float("nan")
        s.req_v[0, reqs[1].block_table[-1], 0, 11] = float("inf")   # key 299, the last row's own

    opt = dict(split_tiles=split, window=25, n_sinks=2)
    sess, _, q, out, lse = run_attn(sh, reqs, n, 5, poison=poison, attn_kernel=2, **opt)
    many, mlse = copied(sess, reqs, q, **opt)
    assert torch.isinf(out[-1]).all() and torch.isfinite(out[4:-1]).all()
    for a, b in ((many, out), (mlse, lse)):
        assert same_bits(a)
        assert torch.equal(torch.isnan(a[0]), torch.isnan(b))
        assert torch.equal(torch.isposinf(a[0]), torch.isposinf(b))
        assert torch.equal(torch.isneginf(a[0]), torch.isneginf(b))


# ------------------------------------------------- the operators as used
def test_decode_after_composed_prefill():
    """A composed prefill, then tokens decoded over its pages: bf16, and from
    4-bit pages, with a window; every output against the oracle."""
    wl = workloads.generate("small_bf16")
    extra = 5
    for r in wl.requests:       # room for the new tokens
        need = -(-(r.prompt_len + extra) // 16) - len(r.block_table)
        r.block_table = np.concatenate([r.block_table, np.arange(
            wl.n_req_pages, wl.n_req_pages + need, dtype=np.int32)]).astype(np.int32)
        wl.n_req_pages += need
    m = wl.model
    sess = Session(m, wl.n_pool_pages, wl.n_req_pages, four_bit=True)
    staging.upload_pool(sess, wl)
    plan = sess.plan(wl.requests)
    q, k, v = staging.fresh_inputs(sess, wl, plan)
    out, lse = sess.new_outputs(plan)
    sess.assemble(plan, k, v)
    sess.attn(plan, q, out, lse)
    reqs = [NS(kv_len=r.prompt_len, n_rows=0, positions=None, row_lo=None,
               block_table=r.block_table.tolist()) for r in wl.requests]
    sess.pack_step(sess.step(reqs, four_bit=True))
    g = gen(11)
    wq, wk = rand(g, 128), rand(g, 128)
    for t in range(extra):
        for r in reqs:
            r.kv_len, r.n_rows = r.kv_len + 1, 1
        T = len(reqs)
        q, k, v = rand(g, T, 32, 128), rand(g, T, 8, 128), rand(g, T, 8, 128)
        for four in (False, True):
            opt = dict(window=48, n_sinks=4) if t % 2 else {}
            step = sess.step(reqs, four_bit=four, **opt)
            q_out, out = torch.empty_like(q), torch.empty_like(q)
            lse = torch.empty(T, 32, device="cuda")
            sess.step_append(step, q, k, v, q_out, None, wq, wk, EPS)
            sess.step_attn(step, q_out, out, lse)
            torch.cuda.synchronize()
            check_attn(reqs, q_out, out, lse, (four_bit_kv if four else pages_kv)(sess, reqs),
                       128, 2000, **opt)


def test_composed_rows_equal_the_plan_attention():
    """A step of a composed prompt's rows (local scope) gives tsr_attn's
    outputs, to both kernels' tolerances."""
    cfg = workloads.get_config("small_bf16").with_(miss_scope="local")
    wl = workloads.make_workload(cfg)
    sess = Session(wl.model, wl.n_pool_pages, wl.n_req_pages)
    staging.upload_pool(sess, wl)
    plan = sess.plan(wl.requests)
    q, k, v = staging.fresh_inputs(sess, wl, plan)
    sess.assemble(plan, k, v)
    pos, r = plan.compute_positions()
    lo = plan.row_kv_lo()
    reqs = [NS(kv_len=x.prompt_len, n_rows=int((r == i).sum()), positions=pos[r == i].tolist(),
               row_lo=lo[r == i].tolist(), block_table=x.block_table.tolist())
            for i, x in enumerate(wl.requests)]
    step = sess.step(reqs)
    k_after = sess.req_k.clone()
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(q.shape[:2], device="cuda")
    sess.step_append(step, q, k, v, q_out)          # no norm: append's own work again
    torch.cuda.synchronize()
    # (bits: unused slots may hold NaN)
    assert torch.equal(sess.req_k.view(torch.int16), k_after.view(torch.int16))
    sess.step_attn(step, q_out, out, lse)
    out2, lse2 = sess.new_outputs(plan)
    sess.attn(plan, q, out2, lse2)
    torch.cuda.synchronize()
    check_attn(reqs, q_out, out, lse, pages_kv(sess, reqs), 128, 2000, part=part_of(step))
    assert (lse - lse2).abs().max() < 1e-4
    assert ((out - out2).float().norm() / out2.float().norm()) < 4e-3


@pytest.mark.parametrize("kernel", [1, 2])
def test_out_in_place_and_shared_prefix(kernel):
    """out may be q; requests may share the pages of a common prefix, also
    when the pages after it are appended to."""
    sh = shape(8, 2)
    reqs, n = batch([(70, 3), (50, 2)], 16)
    reqs[1].block_table = reqs[0].block_table[:2] + reqs[1].block_table[2:]
    sess, step, q, out, lse = run_attn(sh, reqs, n, 21, attn_kernel=kernel, split_tiles=1)
    # (run_attn wrote the shared pages for each request: what is there now)
    K = pages_kv(sess, reqs)
    k, v = rand(gen(1), 5, 2, 128), rand(gen(2), 5, 2, 128)
    q_out = torch.empty_like(q)
    sess.step_append(step, q, k, v, q_out)
    lse = torch.empty(5, 8, device="cuda")
    out = q_out.clone()
    sess.step_attn(step, out, out, lse)
    torch.cuda.synchronize()
    check_attn(reqs, q_out, out, lse, K, 128, 70, part=part_of(step))


def test_captured_step_replays():
    """append + attention captured in a graph, replayed on new inputs with
    eager work between the replays."""
    sh = shape(8, 2)
    reqs, n = batch([(200, 1), (90, 1), (33, 2)], 16)
    sess = Session(sh, 1, n)
    g = gen(8)
    sess.req_k[0], sess.req_v[0] = rand(g, n, 2, 16, 128), rand(g, n, 2, 16, 128)
    step = sess.step(reqs, split_tiles=2, window=60, n_sinks=3)
    assert step.num_attn_splits > 0
    T = step.num_rows
    q, k, v, w = rand(g, T, 8, 128), rand(g, T, 2, 128), rand(g, T, 2, 128), rand(g, 128)
    q_out, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(T, 8, device="cuda")

    def layer(stream, q_out, out, lse):
        sess.step_append(step, q, k, v, q_out, None, w, w, EPS, stream=stream)
        sess.step_attn(step, q_out, out, lse, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer(torch.cuda.current_stream(), q_out, out, lse)
    for seed in range(4):
        for t in (q, k, v):
            t.copy_(rand(gen(seed), *t.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (q_out, out, lse)]
        e = [torch.empty_like(x) for x in (q_out, out, lse)]
        layer(None, *e)
        torch.cuda.synchronize()
        for a, b in zip(got, e):
            assert torch.equal(a, b)


def test_one_step_on_two_streams():
    """A step without cut ranges serves two streams at once."""
    sh = shape(8, 2)
    reqs, n = batch([(400, 1), (90, 20)], 16)
    sess, step, q, out, lse = run_attn(sh, reqs, n, 12, split_tiles=-1)
    assert step.num_attn_splits == 0
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [torch.empty_like(out) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o in zip(streams, outs):
            sess.step_attn(step, q, o, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, out)


@pytest.mark.parametrize("handle", [False, True])
def test_step_of_a_stream(handle):
    """A step made for a stream other than the current one, between other work
    on either, with its workspace in memory freed on the current one."""
    sh = shape(8, 2)
    reqs, n = batch([(700, 1), (90, 1)], 16)
    sess, step, q, out, lse = run_attn(sh, reqs, n, 21, split_tiles=2)
    assert step.num_attn_splits > 0
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(3):
        junk = torch.full((step.workspace.numel(),), i, dtype=torch.uint8, device="cuda")
        for _ in range(20):
            junk.add_(1)
        del junk   # free for the current stream only
        other = sess.step(reqs, stream=side.cuda_stream if handle else side, split_tiles=2)
        o, l = torch.empty_like(out), torch.empty_like(lse)
        side.wait_stream(torch.cuda.current_stream())
        sess.step_attn(other, q, o, l, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(l, lse)


# ---------------------------------------------------------------- refusals
def test_calls_refused_before_any_launch():
    sh = shape(8, 2)
    reqs, n = batch([(40, 1), (20, 1)], 16)
    reqs.append(NS(kv_len=40, n_rows=0, positions=None, row_lo=None,
                   block_table=reqs[0].block_table))      # shares the page appended to
    sess = Session(sh, 1, n, four_bit=True)
    step, step4 = sess.step(reqs), sess.step(reqs[:2], four_bit=True)
    own = sess.step(reqs[:2])
    q = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    rk, rv, r4 = sess.req_k[0], sess.req_v[0], sess.req4_scale[0]

    def bad(match, f, *a, **kw):
        with pytest.raises(P.TsrError, match=match) as e:
            f(*a, **kw)
        assert e.value.status == P.TSR_ERR_INVALID_ARG

    ap, at = P.tsr_step_append, P.tsr_step_attn
    bad("block table twice", ap, step, q, k, k, rk, rv, None, q)
    bad("4-bit pages only", ap, own, q, k, k, rk, rv, r4, q)
    bad("need their scale", ap, step4, q, k, k, rk, rv, None, q)
    bad("4-bit pages only", at, own, q, rk, rv, r4, q)
    bad("need their scale", at, step4, q, rk, rv, None, q)
    for i in (1, 2, 3, 4, 5, 7):
        a = [own, q, k, k, rk, rv, None, q.clone()]
        a[i] = None
        bad("NULL", ap, *a)
    for i in (1, 2, 3, 5):
        a = [own, q, rk, rv, None, q.clone()]
        a[i] = None
        bad("NULL", at, *a)
    bad("aligned", ap, own, q.data_ptr() + 8, k, k, rk, rv, None, q)
    bad("aligned", at, own, q, rk.data_ptr() + 2, rv, None, q.clone())
    bad("aligned", at, own, q, rk, rv, None, q.clone(), 4098)
    bad("strides", ap, own, q, k, k, rk, rv, None, q.clone(), q_stride=1016)
    bad("strides", ap, own, q, k, k, rk, rv, None, q.clone(), k_stride=260)
    bad("strides", ap, own, q, k, k, rk, rv, None, q.clone(), v_stride=-256)
    bad("only if those are packed", ap, own, q, k, k, rk, rv, None, q, q_stride=2048)
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        bad("eps", ap, own, q, k, k, rk, rv, None, q, norm=P.make_qk_norm(eps=eps))
    bad("aligned", ap, own, q, k, k, rk, rv, None, q,
        norm=P.make_qk_norm(q_weight=q.data_ptr() + 2))
    bad("E2M1", P.tsr_step_pack_kv, own, rk, rv, rk, rv, r4)
    bad("E2M1", P.tsr_step_unpack_kv, own, rk, rv, r4, rk, rv)
    bad("NULL", P.tsr_step_pack_kv, step4, rk, rv, rk, None, r4)
    # a session checks shapes and types too
    for f in (lambda: sess.step_attn(own, q[:1], q), lambda: sess.step_attn(own, q.float(), q),
              lambda: sess.step_append(own, q, k.transpose(1, 2), k, q),
              lambda: sess.step_append(own, q, k, k, q, q_weight=k[0, 0]),
              lambda: sess.step_attn(own, q, q.clone(), torch.empty(2, 8, device="cuda").double()),
              lambda: Session(sh, 1, n).step(reqs, four_bit=True)):
        with pytest.raises(ValueError):
            f()
    torch.cuda.synchronize()


def test_no_rows_is_no_work():
    sess = Session(shape(), 1, 4, four_bit=True)
    s = sess.step([])
    e = torch.empty(0, 8, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.empty(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    sess.step_append(s, e, k, k, e)
    sess.step_attn(s, e, e)
    sess.pack_step(sess.step([], four_bit=True))
    torch.cuda.synchronize()
