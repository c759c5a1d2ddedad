"""Policy and preference loss on logits against their definitions in 64 bits, against differences, and at the sizes,
masks, strides and alignments where they can go wrong."""

import pytest
import torch

from tests import llm_reference as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda"


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def difference(f, h):
    """The derivative of f at 0 from four values: the error is of the order of h^4 times the fifth derivative."""
    v = [float(f(s * h).double()) for s in (1, -1, 2, -2)]
    return (8 * (v[0] - v[1]) - (v[2] - v[3])) / (12 * h)


def policy_case(T, V, dtype, seed, spread=2.0):
    g = gen(seed)
    z = (torch.randn(T, V, generator=g, device=DEV) * spread).to(DT[dtype])
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    logp = R.rows_logp(z, y)[0].float().to(DEV)
    old = logp + 0.3 * torch.randn(T, generator=g, device=DEV)
    # no ratio within 1e-4 of a bound of the clip, where the gradient jumps
    for b in (0.8, 1.2):
        r = torch.exp(logp - old)
        old = torch.where((r - b).abs() < 1e-4, old - 5e-3, old)
    ref = logp + 0.5 * torch.randn(T, generator=g, device=DEV)
    adv = torch.randn(T, generator=g, device=DEV)
    w = torch.rand(T, generator=g, device=DEV) / T
    return z, y, old, adv, w, ref


def check_policy(r, want, z, kl_coef, need_grad=True):
    e = R.logp_error(z, want["logp"])
    live = want["live"].to(R.D)
    R.close(r.logp, want["logp"], e * live, "logp")
    size = want["size"]
    R.close(r.loss[None], want["loss"][None], (size * (e + 1e-6)).sum()[None], "loss")
    R.close(r.kl[None], want["kl"][None], (want["kl_size"] * (e + 1e-6)).sum()[None], "kl")
    R.close(r.clipped[None], want["clipped"][None], want["clipped"].abs()[None] * 1e-6, "clipped")
    if need_grad:
        # g has the error of its terms, softmax_v that of exp and 1 / S (2 e covers both), each element is below |g| in size
        R.close(r.dlogits, want["dlogits"], ((size * (e + 1e-6)) + 2 * e * size)[:, None], "dlogits")


SHAPES = [(1, 1), (3, 2), (5, 31), (4, 32), (9, 33), (7, 255), (17, 1000), (5, 1024), (3, 1025), (6, 4097), (1, 32000), (3, 50257), (2, 151936), (300, 2049),
          (1, 300001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", SHAPES)
def test_policy_loss_and_gradient(llm, T, V, dtype):
    z, y, old, adv, w, ref = policy_case(T, V, dtype, T * 131 + V)
    for kl_coef, rf in ((0.0, None), (0.07, ref)):
        r = llm.policy_loss(z, y, old, adv, w, logp_ref=rf, kl_coef=kl_coef)
        check_policy(r, R.policy(z, y, old, adv, w, rf, kl_coef=kl_coef), z, kl_coef)
    only = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.07, need_grad=False)
    assert only.dlogits is None and torch.equal(only.loss, r.loss) and torch.equal(only.logp, r.logp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 3001, 20000])
def test_policy_strides_alignments_and_in_place(llm, V, dtype):
    T = 11
    z, y, old, adv, w, ref = policy_case(T, V, dtype, V)
    want = R.policy(z, y, old, adv, w, ref, kl_coef=0.1)
    for left, right in ((0, 0), (1, 0), (3, 5), (8, 8), (0, 1), (5, 0)):
        big = torch.full((T, V + left + right), float("nan"), dtype=z.dtype, device=DEV)
        big[:, left:left + V] = z
        view = big[:, left:left + V]
        for oleft in (left, 0, 2):
            obig = torch.full((T, V + 9), 7.0, dtype=z.dtype, device=DEV)
            out = obig[:, oleft:oleft + V]
            r = llm.policy_loss(view, y, old, adv, w, logp_ref=ref, kl_coef=0.1, dlogits=out)
            check_policy(r, want, z, 0.1)
            assert r.dlogits.data_ptr() == out.data_ptr()
            assert (obig[:, :oleft] == 7).all() and (obig[:, oleft + V:] == 7).all()
        r = llm.policy_loss(view, y, old, adv, w, logp_ref=ref, kl_coef=0.1, dlogits=view)      # in place
        check_policy(r, want, z, 0.1)
        assert torch.isnan(big[:, :left]).all() and torch.isnan(big[:, left + V:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [37, 2500, 33000])
def test_policy_masks(llm, V, dtype):
    """Left-out tokens hold NaN and infinities, kept rows have -inf and the type's lowest value, some are banned entirely."""
    T = 24
    z, y, old, adv, w, ref = policy_case(T, V, dtype, V + 1)
    low = torch.finfo(z.dtype).min
    at = torch.arange(T, device=DEV)
    zy = z[at, y.long()].clone()
    z[0:4] = torch.where(torch.rand(4, V, generator=gen(3), device=DEV) < 0.9, torch.full_like(z[:4], float("-inf")), z[:4])
    z[4:8] = torch.where(torch.rand(4, V, generator=gen(4), device=DEV) < 0.9, torch.full_like(z[:4], low), z[4:8])
    z[at, y.long()] = zy
    z[8] = float("-inf")                 # nothing is left of this row
    z[9] = low                           # a row of the lowest value: uniform
    z[10] = float("-inf")
    z[10, y[10].long()] = 1.5            # one token is left: logp 0, gradient 0
    z[11] = float("nan")
    z[12] = float("inf")
    z[13] = float("nan")
    w[11] = 0.0
    y[12] = -100
    y[13] = V
    w[14] = 0.0
    old[8:14] = 0.0
    ref[8:14] = 0.0
    old[9] = ref[9] = -float(torch.log(torch.tensor(float(V))))
    r = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1)
    clean = z.clone()
    clean[11:14] = 0
    want = R.policy(clean, torch.where((torch.arange(T, device=DEV) == 12) | (torch.arange(T, device=DEV) == 13), torch.full_like(y, -1), y), old, adv, w, ref, kl_coef=0.1)
    check_policy(r, want, clean, 0.1)
    for t in (8, 11, 12, 13, 14):
        assert (r.dlogits[t] == 0).all() and r.logp[t] == 0
    zero = llm.policy_loss(z, y, old, adv, torch.zeros_like(w), logp_ref=ref, kl_coef=0.1)      # every token is left out
    assert zero.loss == 0 and zero.kl == 0 and (zero.dlogits == 0).all() and (zero.logp == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(200, 1500), (160, 5001), (90, 40000), (80, 70001)])
def test_many_rows(llm, T, V, dtype):
    """More rows than half the SMs: rows that one warp takes, rows within and beyond what stays in shared memory; some are left
    out; in place and beside."""
    z, y, old, adv, w, ref = policy_case(T, V, dtype, T + V)
    w[::5] = 0.0
    y[3::11] = -1
    z[::5] = float("nan")
    clean = torch.nan_to_num(z)
    want = R.policy(clean, y, old, adv, w, ref, kl_coef=0.1)
    a = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1)
    check_policy(a, want, clean, 0.1)
    only = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1, need_grad=False)
    assert torch.equal(only.loss, a.loss) and torch.equal(only.logp, a.logp)
    lens = (T // 4, T // 3, 0, T - T // 4 - T // 3)
    off = torch.tensor([0, lens[0], lens[0] + lens[1], lens[0] + lens[1], T], dtype=torch.int32, device=DEV)
    yy = torch.where(w == 0, torch.full_like(y, -100), y)
    sums = R.preference(clean, yy, off, torch.zeros(4))["seq_logp"].float().to(DEV)
    sref = sums + torch.tensor([3.0, -2.0, 0.0, 1.0], device=DEV)
    p = llm.preference_loss(z, yy, off, sref, beta=0.2)
    check_pref(p, R.preference(clean, yy, off, sref, 0.2), clean, 0.2, 0.5)
    q = llm.preference_loss(z.clone(), yy, off, sref, beta=0.2, need_grad=False)
    assert torch.equal(q.loss, p.loss) and torch.equal(q.pair_loss, p.pair_loss)
    spare = z.clone()
    p2 = llm.preference_loss(spare, yy, off, sref, beta=0.2, dlogits=spare)
    assert torch.equal(p2.dlogits, p.dlogits)
    b = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1, dlogits=z)
    for u, v in zip(a, b):
        assert torch.equal(u, v)


def test_policy_nan_in_a_kept_row_is_not_hidden(llm):
    for V in (50, 5000, 40000):
        z, y, old, adv, w, ref = policy_case(4, V, "f32", 5)
        z[2, V // 2] = float("nan")
        r = llm.policy_loss(z, y, old, adv, w)
        assert torch.isnan(r.loss) and torch.isnan(r.dlogits[2]).all() and torch.isfinite(r.dlogits[[0, 1, 3]]).all()


def test_policy_clip_branches(llm):
    """One token on each side of each bound, for either sign of the advantage."""
    V = 64
    z, y, *_ = policy_case(8, V, "f32", 9)
    logp = R.rows_logp(z, y)[0].float().to(DEV)
    shift = torch.tensor([0.5, 0.5, -0.5, -0.5, 0.1, 0.1, -0.1, -0.1], device=DEV)
    adv = torch.tensor([2.0, -2.0, 2.0, -2.0, 2.0, -2.0, 2.0, -2.0], device=DEV)
    w = torch.full((8,), 0.125, device=DEV)
    r = llm.policy_loss(z, y, logp - shift, adv, w, clip_low=0.2, clip_high=0.3)
    want = R.policy(z, y, logp - shift, adv, w, lo=0.2, hi=0.3)
    check_policy(r, want, z, 0.0)
    rows_of_zeros = (r.dlogits == 0).all(1).tolist()
    assert rows_of_zeros == [True, False, False, True, False, False, False, False]
    assert float(r.clipped) == 0.25
    # an advantage of zero counts for nothing whatever the ratio is
    none = llm.policy_loss(z, y, logp - 1000.0, torch.zeros(8, device=DEV), w)
    assert none.loss == 0 and (none.dlogits == 0).all()


@pytest.mark.parametrize("V", [17, 3000])
def test_policy_gradient_against_differences(llm, V):
    T = 6
    z, y, old, adv, w, ref = policy_case(T, V, "f32", 77)
    w = w * 0 + 1.0 / T
    adv = adv.clamp(-1.5, 1.5)
    # far from the clip's corners: a step must not cross one
    logp = R.rows_logp(z, y)[0].float().to(DEV)
    old = logp + torch.tensor([0.05, -0.05, 0.5, -0.5, 0.0, 0.6], device=DEV)
    kw = dict(logp_ref=ref, kl_coef=0.1)
    r = llm.policy_loss(z, y, old, adv, w, **kw)
    step = 2e-2
    for k in range(4):
        v = torch.randn(T, V, generator=gen(k), device=DEV)
        v[torch.arange(T, device=DEV), y.long()] *= 3
        diff = difference(lambda s: llm.policy_loss(z + s * v, y, old, adv, w, **kw).loss, step)
        slope = float((r.dlogits.double() * v.double()).sum())
        # the loss is of order 1 (error below 1e-5, over the step: 1e-3 at most)
        assert abs(diff - slope) <= 3e-3 + 1e-3 * abs(slope), (k, diff, slope)


def pref_case(lens, V, dtype, seed, prompt=0):
    g = gen(seed)
    T = sum(lens)
    z = (torch.randn(T, V, generator=g, device=DEV) * 2).to(DT[dtype])
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    at = torch.tensor([0] + list(lens)).cumsum(0)
    for a, b in zip(at[:-1].tolist(), at[1:].tolist()):
        y[a:min(b, a + prompt)] = -100
    offsets = at.to(torch.int32).to(DEV)
    s = R.preference(z, y, offsets, torch.zeros(len(lens)))["seq_logp"].float().to(DEV)
    return z, y, offsets, s + 5 * torch.randn(len(lens), generator=g, device=DEV)


def check_pref(r, want, z, beta, scale, need_grad=True):
    e = R.logp_error(z, want["logp"])
    at = want["at"]
    es = torch.stack([e[a:max(a, b)].sum() for a, b in zip(at[:-1], at[1:])]) if len(at) > 1 else torch.zeros(0, dtype=R.D)
    R.close(r.seq_logp, want["seq_logp"], es, "seq_logp")
    eh = beta * (es[0::2] + es[1::2])
    R.close(r.pair_loss, want["pair_loss"], eh + 1e-7, "pair_loss")           # |d loss / d h| <= 1
    R.close(r.loss[None], want["loss"][None], scale * (eh + 1e-7 + want["pair_loss"] * 2e-7).sum()[None], "loss")
    if need_grad:
        # |d g / d h| <= scale beta / 4; softmax's own error relative to |g|
        eg = torch.zeros(z.shape[0], dtype=R.D)
        for q in range(len(at) - 1):
            eg[at[q]:max(at[q], at[q + 1])] = scale * beta * (eh[q // 2] / 4 + 1e-7)
        R.close(r.dlogits, want["dlogits"], (eg + 3 * e * want["g"].abs())[:, None], "dlogits")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,V,prompt", [
    ((1, 1), 1, 0), ((3, 2), 2, 0), ((4, 0), 33, 0), ((0, 0), 40, 0), ((5, 7, 1, 9), 1000, 2), ((6, 3), 1025, 6), ((33, 20), 32000, 8),
    ((17, 1, 0, 40, 3, 3), 4099, 1), ((2, 3), 50257, 1), ((1, 2), 151936, 0), ((200, 300), 777, 10),
])
def test_preference_loss_and_gradient(llm, lens, V, prompt, dtype):
    z, y, off, ref = pref_case(lens, V, dtype, V + len(lens), prompt)
    for smoothing, scale in ((0.0, None), (0.1, 0.37)):
        r = llm.preference_loss(z, y, off, ref, beta=0.2, smoothing=smoothing, scale=scale)
        want = R.preference(z, y, off, ref, 0.2, smoothing, scale)
        check_pref(r, want, z, 0.2, 2.0 / len(lens) if scale is None else scale)
    only = llm.preference_loss(z, y, off, ref, beta=0.2, smoothing=0.1, scale=0.37, need_grad=False)
    assert only.dlogits is None and torch.equal(only.loss, r.loss) and torch.equal(only.seq_logp, r.seq_logp)
    same = llm.preference_loss(z, y, off, ref, beta=0.2, smoothing=0.1, scale=0.37, dlogits=z)          # in place
    assert torch.equal(same.dlogits, r.dlogits) and torch.equal(same.loss, r.loss)


def test_preference_rows_outside_answers_and_bad_offsets(llm):
    V = 1500
    z, y, off, ref = pref_case((5, 6, 4, 7), V, "f32", 3, 1)
    z[-2:] = float("nan")
    z[0] = float("-inf")
    off = off.clone()
    off[-1] -= 2                                            # the last two rows belong to no answer
    y[-2:] = -1
    y[1] = V + 5
    r = llm.preference_loss(z, y, off, ref)
    clean = z.clone()
    clean[-2:] = 0
    check_pref(r, R.preference(clean, y, off, ref), clean, 0.1, 0.5)
    assert (r.dlogits[-2:] == 0).all() and (r.dlogits[:2] == 0).all()
    wild = torch.tensor([-7, 5, 3, 15, 1000000], dtype=torch.int32, device=DEV)         # clamped; a descending pair is empty
    clean = torch.where(torch.isfinite(z), z, torch.zeros((), device=DEV))
    r = llm.preference_loss(clean, y, wild, ref)
    s = r.seq_logp
    assert s[1] == 0 and torch.isfinite(r.loss)


def test_preference_extreme_margins(llm):
    """Margins far beyond exp's range: the loss is linear or zero there, never infinite or NaN."""
    z, y, off, ref = pref_case((4, 4, 4, 4), 100, "f32", 11)
    s = R.preference(z, y, off, ref)["seq_logp"].float().to(DEV)
    ref = s + torch.tensor([1e5, 0.0, 0.0, 1e5], device=DEV)
    r = llm.preference_loss(z, y, off, ref, beta=1.0)
    want = R.preference(z, y, off, ref, 1.0)
    check_pref(r, want, z, 1.0, 0.5)
    assert abs(float(r.pair_loss[0]) - 1e5) < 1 and float(r.pair_loss[1]) == 0


def test_preference_gradient_against_differences(llm):
    T, V = 10, 200
    z, y, off, ref = pref_case((6, 4), V, "f32", 21, 1)
    r = llm.preference_loss(z, y, off, ref, beta=0.5, smoothing=0.05)
    step = 2e-2
    for k in range(4):
        v = torch.randn(T, V, generator=gen(k), device=DEV)
        diff = difference(lambda s: llm.preference_loss(z + s * v, y, off, ref, beta=0.5, smoothing=0.05).loss, step)
        slope = float((r.dlogits.double() * v.double()).sum())
        assert abs(diff - slope) <= 3e-3 + 1e-3 * abs(slope), (k, diff, slope)


def test_no_tokens(llm):
    f = lambda n: torch.zeros(n, device=DEV)  # noqa: E731
    y = torch.zeros(0, dtype=torch.int32, device=DEV)
    r = llm.policy_loss(torch.zeros(0, 8, device=DEV), y, f(0), f(0), f(0))
    assert r.loss == 0 and r.kl == 0 and r.clipped == 0 and r.dlogits.shape == (0, 8)
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    r = llm.preference_loss(torch.zeros(0, 8, device=DEV), y, off, f(2))
    assert abs(float(r.loss) - 0.6931472) < 1e-6 and (r.seq_logp == 0).all()
    r = llm.preference_loss(torch.zeros(0, 8, device=DEV), y, torch.zeros(1, dtype=torch.int32, device=DEV), f(0))
    assert r.loss == 0


def test_rows_beyond_two_gigaelements(llm):
    """The last row starts more than 2^31 elements behind the first."""
    T, V, ld = 3, 1030, 1_200_000_000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    store = torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device=DEV)
    view = store.as_strided((T, V), (ld, 1))
    z, y, old, adv, w, ref = policy_case(T, V, "bf16", 2)
    view.copy_(z)
    r = llm.policy_loss(view, y, old, adv, w, dlogits=view)
    check_policy(r, R.policy(z, y, old, adv, w), z, 0.0)
    del store, view, r
    torch.cuda.empty_cache()


def test_equal_inputs_give_equal_bits_on_any_stream(llm):
    z, y, old, adv, w, ref = policy_case(700, 3000, "bf16", 1)
    a = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1)
        zp, yp, off, rf = pref_case((30, 20, 9, 50), 2000, "f32", 6)
        p = llm.preference_loss(zp, yp, off, rf)
    s.synchronize()
    q = llm.preference_loss(zp, yp, off, rf)
    for u, v in zip(a + p, b + q):
        assert torch.equal(u, v)
