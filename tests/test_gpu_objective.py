"""GPU parity of the policy and preference losses through the C ABI, against
the fp64 oracle.

Tolerances.  A token's derivative is made of one fp32 difference, exp or
expm1 (2 ulp), and a few products: 2e-6 of its terms' magnitudes.  The loss
adds such terms in pairs of fp32 (48 bits): 2e-6 of the sum of magnitudes.  The
preference loss is computed in such pairs from exact differences and rounded:
1e-6.  dh is rounded to bf16 once: 2^-8 of the element."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle.objective_oracle import MEAN_SEQS, MEAN_TOKENS, SIGMOID, SUM
from paper_2606_19528_gb300 import lora
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

NAN = float("nan")


def f32(a):
    return torch.tensor(np.asarray(a, np.float32), device="cuda")


class Tokens:
    """Flat sequences with a masked prompt each; what is masked holds NaN everywhere but in the mask."""

    def __init__(self, seed, lens, d=64, prompt=0.3, masked=True, junk=True):
        g = np.random.default_rng(seed)
        self.lens, self.d = list(lens), d
        self.off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.T = T = int(self.off[-1])
        self.nll = g.exponential(1.0, T).astype(np.float32)
        self.old = (self.nll + 0.25 * g.standard_normal(T)).astype(np.float32)
        self.ref = (self.nll + 0.25 * g.standard_normal(T)).astype(np.float32)
        self.mask = np.ones(T, np.uint8)
        if masked:
            for a, n in zip(self.off, lens):
                self.mask[a:a + int(prompt * n)] = 0
            self.mask[g.random(T) < 0.1] = 0
        self.dev = {k: f32(np.where((self.mask == 0) & junk, np.nan, getattr(self, k)))
                    for k in ("nll", "old", "ref")}
        self.dh_nll = torch.tensor(g.standard_normal((T, d)), device="cuda").to(torch.bfloat16)
        self.dh64 = G.host_f64(self.dh_nll)
        if junk:
            self.dh_nll[torch.tensor(self.mask == 0, device="cuda")] = NAN
        self.dmask = torch.tensor(self.mask, device="cuda") if masked else None
        self.doff = torch.tensor(self.off, device="cuda")
        self.loss = torch.full((3,), NAN, device="cuda")
        self.w = torch.full((T + 2,), 55.0, device="cuda")
        self.dh = torch.full((T + 1, d), 55.0, device="cuda", dtype=torch.bfloat16)

    def outputs(self):
        return dict(dh_nll=self.dh_nll, dh=self.dh, token_weight=self.w[1:])

    def check_rows(self, w):
        got = G.host_f64(self.dh[:self.T])
        want = w[:, None] * self.dh64
        assert (got[w == 0] == 0).all()
        # the row's weight is the fp32 one that the call returned
        w32 = self.w[1:self.T + 1].double().cpu().numpy()
        assert (np.abs(got - w32[:, None] * self.dh64) <= 2.0 ** -8 * np.abs(want) + 1e-30).all()
        assert (self.dh[self.T:] == 55).all() and self.w[0] == 55 and self.w[-1] == 55 and torch.isnan(
            self.loss[1:]).all()


def call(fn, size, args, junk=0x7f):
    n = size(args)
    ws = torch.full((n + 256,), junk, dtype=torch.uint8, device="cuda")
    fn(args, ws, n)
    torch.cuda.synchronize()
    assert (ws[n:] == junk).all()


def policy(t, adv, kl, low=0.2, high=0.25, beta=0.07, scale=1.3, reduction=MEAN_TOKENS, status=lora.LORA_OK, **kw):
    per_token = len(adv) == t.T and len(adv) != len(t.lens)
    stats = torch.full((2,), NAN, device="cuda")
    out = t.outputs()
    out.update(kw)
    t.adv = f32(adv)  # the arguments hold addresses only
    args = lora.make_policy_args(t.T, len(t.lens), t.d, t.doff, t.dev["nll"], t.dev["old"], t.adv, t.loss,
                                 ref_nll=t.dev["ref"] if kl else None, mask=t.dmask, advantage_per_token=per_token,
                                 clip_low=low, clip_high=high, beta=beta, scale=scale, reduction=reduction,
                                 stats=stats, **out)
    call(lora.lora_policy_fwd_bwd, lora.lora_policy_workspace_size, args)
    assert lora.lora_read_status() == status
    return stats


def check_policy(t, adv, kl, low=0.2, high=0.25, beta=0.07, scale=1.3, reduction=MEAN_TOKENS, rows=True):
    stats = policy(t, adv, kl, low, high, beta, scale, reduction)
    low, high, beta, scale = (float(np.float32(v)) for v in (low, high, beta, scale))
    adv = np.asarray(adv, np.float32)
    loss, w, kl_mean, share = oracle.policy_loss(t.nll, t.old, t.ref if kl else None, adv, t.mask, t.off, low, high,
                                                 beta, scale, reduction)
    # magnitudes: every term without its sign
    rho = np.exp(t.old.astype(np.float64) - t.nll)
    e = t.nll.astype(np.float64) - t.ref
    seq = np.repeat(np.arange(len(t.lens)), t.lens)
    a = np.abs(adv if len(adv) == t.T and len(adv) != len(t.lens) else adv[seq])
    on = t.mask != 0
    n_all = max(int(on.sum()), 1)
    n_seq = np.array([max(int(on[i:j].sum()), 1) for i, j in zip(t.off, t.off[1:])])
    norm = {SUM: np.ones(t.T), MEAN_TOKENS: np.full(t.T, 1 / n_all),
            MEAN_SEQS: 1 / (len(t.lens) * n_seq[seq])}[reduction] * abs(scale)
    size_w = norm * (a * rho + (beta * (np.exp(e) + 1) if kl else 0))
    size_l = float((norm * (a * rho + (beta * (np.abs(np.expm1(e)) + np.abs(e)) if kl else 0)))[on].sum())
    got = t.w[1:t.T + 1].double().cpu().numpy()
    assert (np.abs(got - w) <= 2e-6 * size_w).all(), np.max(np.abs(got - w) / size_w)
    assert abs(float(t.loss[0]) - loss) <= 2e-6 * size_l + 1e-30
    assert float(stats[0]) == pytest.approx(kl_mean, rel=3e-6, abs=1e-12)
    assert float(stats[1]) == pytest.approx(share, rel=1e-6)
    if rows:
        t.check_rows(w)


@pytest.mark.parametrize("reduction", [SUM, MEAN_TOKENS, MEAN_SEQS])
@pytest.mark.parametrize("kl", [False, True])
@pytest.mark.parametrize("per_token", [False, True])
def test_policy(reduction, kl, per_token):
    t = Tokens(1, [5, 0, 131, 1, 700, 64, 0])
    adv = np.random.default_rng(2).standard_normal(t.T if per_token else len(t.lens))
    check_policy(t, adv, kl, reduction=reduction)


@pytest.mark.parametrize("lens", [[1], [2], [0, 1], [33, 0], [4097], [1] * 300, [20000, 3], list(range(40))])
@pytest.mark.parametrize("reduction", [MEAN_TOKENS, MEAN_SEQS])
def test_policy_lengths(lens, reduction):
    t = Tokens(len(lens), lens, d=8, prompt=0.5)
    check_policy(t, np.random.default_rng(3).standard_normal(len(lens)), True, reduction=reduction)


@pytest.mark.parametrize("d", [8, 16, 248, 256, 264, 1024, 2056, 11008])
def test_policy_row_widths(d):
    t = Tokens(d, [7, 30], d=d)
    check_policy(t, [1.0, -0.5], True)


def test_policy_without_mask_and_without_rows():
    t = Tokens(4, [50, 20, 9], masked=False, junk=False)
    check_policy(t, [0.5, -2.0, 0.0], True)
    t2 = Tokens(4, [50, 20, 9], masked=False, junk=False)
    policy(t2, [0.5, -2.0, 0.0], True, dh=None, dh_nll=None)
    assert torch.equal(t2.w, t.w) and torch.equal(t2.loss[:1], t.loss[:1]) and (t2.dh == 55).all()
    t3 = Tokens(4, [50, 20, 9], masked=False, junk=False)
    policy(t3, [0.5, -2.0, 0.0], True, dh=None, dh_nll=None, token_weight=None)
    assert torch.equal(t3.loss[:1], t.loss[:1]) and (t3.w == 55).all()
    t4 = Tokens(4, [50, 20, 9], masked=False, junk=False)
    policy(t4, [0.5, -2.0, 0.0], True, dh=t4.dh_nll, token_weight=None)  # in place
    assert torch.equal(t4.dh_nll, t.dh[:t.T])


def test_policy_all_masked():
    for reduction in (SUM, MEAN_TOKENS, MEAN_SEQS):
        t = Tokens(5, [6, 3])
        t.dmask.zero_()
        for v in t.dev.values():
            v.fill_(NAN)
        stats = policy(t, [1.0, 1.0], True, reduction=reduction)
        assert t.loss[0] == 0 and (t.w[1:-1] == 0).all() and (t.dh[:t.T] == 0).all() and (stats == 0).all()


def test_policy_clipped_rows_are_zero_whatever_they_hold():
    t = Tokens(6, [40], masked=False, junk=False)
    t.old = (t.nll + np.where(np.arange(40) % 2, 1.0, 0.0)).astype(np.float32)
    t.dev["old"] = f32(t.old)
    t.dh_nll[1::2] = float("inf")
    policy(t, [1.0], False)
    assert (t.w[2:-1:2] == 0).all() and (t.dh[1:40:2] == 0).all() and (t.dh[0:40:2] != 0).any(dim=1).all()


def test_policy_extreme_values():
    """Ratios that overflow, no lower bound (clip_low 1), a NaN on a trainable token: what IEEE arithmetic gives."""
    t = Tokens(7, [4], masked=False, junk=False)
    t.nll[:] = [0.0, 200.0, 0.0, 1.0]
    t.old[:] = [200.0, 0.0, 1.0, 1.0]
    for k in ("nll", "old"):
        t.dev[k] = f32(getattr(t, k))
    policy(t, [-1.0], False, low=1.0, reduction=SUM, scale=1.0)
    assert t.w[1] == -math.inf and abs(float(t.w[2])) < 1e-30 and float(t.w[3]) == pytest.approx(-math.e)
    t.dev["nll"][3] = NAN
    policy(t, [-1.0], False, low=1.0, reduction=SUM, scale=1.0)
    assert torch.isnan(t.loss[0]) and torch.isnan(t.w[4]) and torch.isnan(t.dh[3]).all()
    assert float(t.w[3]) == pytest.approx(-math.e)


def test_policy_bounds_go_by_the_fp32_difference():
    high = 0.25
    lim = np.float32(math.log1p(high))
    t = Tokens(8, [3], masked=False, junk=False)
    t.nll[:] = 0.0
    t.old[:] = [lim, np.nextafter(lim, np.float32(9)), np.nextafter(lim, np.float32(-9))]
    t.dev["nll"], t.dev["old"] = f32(t.nll), f32(t.old)
    policy(t, [1.0], False, high=high)
    assert [float(v) != 0 for v in t.w[1:4]] == [True, False, True]


@pytest.mark.parametrize("off", [[0, 5, 3, 12], [1, 4, 8, 12], [0, 4, 8, 11], [0, 4, 8, 13], [0, -4, 8, 12],
                                 [0, 4, 2 ** 30, 12]])
def test_policy_offsets_out_of_order_are_reported(off):
    t = Tokens(9, [4, 4, 4])
    t.doff = torch.tensor(off, dtype=torch.int32, device="cuda")
    policy(t, [1.0, 1.0, 1.0], True, status=lora.LORA_EINVAL)
    assert (t.dh[t.T:] == 55).all() and t.w[0] == 55 and t.w[-1] == 55
    assert lora.lora_read_status() == lora.LORA_OK


def pref(t, ref, kind, mean_tokens, beta, margin, smoothing, scale, status=lora.LORA_OK, **kw):
    rewards = torch.full((len(t.lens),), NAN, device="cuda")
    out = t.outputs()
    out.update(kw)
    args = lora.make_pref_args(t.T, len(t.lens) // 2, t.d, t.doff, t.dev["nll"], t.loss,
                               ref_nll=t.dev["ref"] if ref else None, mask=t.dmask, kind=kind,
                               mean_tokens=mean_tokens, beta=beta, margin=margin, label_smoothing=smoothing,
                               scale=scale, rewards=rewards, **out)
    call(lora.lora_pref_fwd_bwd, lora.lora_pref_workspace_size, args)
    assert lora.lora_read_status() == status
    return rewards


def check_pref(t, ref=True, kind=SIGMOID, mean_tokens=False, beta=0.1, margin=0.05, smoothing=0.0, scale=1.3):
    rewards = pref(t, ref, kind, mean_tokens, beta, margin, smoothing, scale)
    beta, margin, smoothing, scale = (float(np.float32(v)) for v in (beta, margin, smoothing, scale))
    loss, w, want = oracle.pref_loss(t.nll, t.ref if ref else None, t.mask, t.off, kind, mean_tokens, beta, margin,
                                     smoothing, scale)
    got = t.w[1:t.T + 1].double().cpu().numpy()
    assert (np.abs(got - w) <= 1e-6 * np.abs(w)).all()
    assert float(t.loss[0]) == pytest.approx(loss, rel=1e-6)
    assert (np.abs(rewards.double().cpu().numpy() - want) <= 1e-6 * np.abs(want) + 1e-12).all()
    t.check_rows(w)


@pytest.mark.parametrize("kind,smoothing", [(0, 0.0), (0, 0.15), (1, 0.0), (2, 0.0)])
@pytest.mark.parametrize("mean_tokens", [False, True])
@pytest.mark.parametrize("ref", [False, True])
def test_pref(kind, smoothing, mean_tokens, ref):
    check_pref(Tokens(20 + kind, [5, 9, 200, 31, 1, 2, 77, 530]), ref, kind, mean_tokens, smoothing=smoothing)


@pytest.mark.parametrize("lens", [[1, 1], [0, 3], [3, 0], [0, 0, 2, 1], [5000, 1], [9000, 9001], [2, 3] * 200])
def test_pref_lengths(lens):
    check_pref(Tokens(len(lens), lens, d=16, prompt=0.4), mean_tokens=len(lens) == 2)


@pytest.mark.parametrize("d", [8, 264, 3000, 11008])
def test_pref_row_widths(d):
    check_pref(Tokens(d, [7, 30], d=d))


@pytest.mark.parametrize("beta", [1.0, 1000.0])
def test_pref_far_from_zero(beta):
    """Margins of hundreds and of over 1e5: no overflow on either side of the sigmoid."""
    for seed in (1, 2):
        t = Tokens(seed, [900, 400] if seed == 1 else [400, 900])
        check_pref(t, ref=False, beta=beta, smoothing=0.1)


def test_pref_without_trainable_tokens():
    t = Tokens(30, [6, 3])
    t.dmask.zero_()
    rewards = pref(t, True, SIGMOID, True, 0.1, 0.0, 0.0, 1.0)
    assert float(t.loss[0]) == pytest.approx(math.log(2.0)) and (rewards == 0).all()
    assert (t.w[1:-1] == 0).all() and (t.dh[:t.T] == 0).all()


def test_pref_offsets_out_of_order_are_reported():
    t = Tokens(9, [4, 4])
    t.doff = torch.tensor([0, 9, 8], dtype=torch.int32, device="cuda")
    pref(t, True, SIGMOID, True, 0.1, 0.0, 0.0, 1.0, status=lora.LORA_EINVAL)
    assert (t.dh[t.T:] == 55).all()


def test_same_bits_every_time_and_on_another_stream():
    t = Tokens(40, [600, 41, 1300, 8])
    adv = [0.3, -1.0, 2.0, 0.1]
    policy(t, adv, True)
    first = [v.clone() for v in (t.loss[:1], t.w, t.dh)]
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            t.dh.zero_()
            policy(t, adv, True)
            t.dh[t.T:] = 55
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (t.loss[:1], t.w, t.dh)))


def test_rows_past_two_to_the_31_elements():
    """1.2 million rows of 2048: byte offsets past 2^32; the rows at the end."""
    T, d = 1200000, 2048
    t = Tokens(50, [T // 2 - 7, T // 2 + 7], d=8, junk=False)
    src = torch.ones(T, d, dtype=torch.bfloat16, device="cuda")
    dh = torch.empty_like(src)
    t.d = d
    policy(t, [1.0, -1.0], True, reduction=SUM, dh_nll=src, dh=dh)
    want = t.w[1:-1].to(torch.bfloat16)
    assert torch.equal(dh[:, 0], want) and torch.equal(dh[:, -1], want) and torch.equal(dh[-3:, 1000], want[-3:])


# Calls on both sides of the number of tokens (256) and of sequences or pairs (32) up to which they are one launch.
@pytest.mark.parametrize("lens", [[5, 0, 31, 1, 100, 64, 0], [256], [257], [8] * 32, [7] * 33, [1] * 31 + [225]])
@pytest.mark.parametrize("reduction", [SUM, MEAN_TOKENS, MEAN_SEQS])
@pytest.mark.parametrize("kl,per_token", [(False, True), (True, False)])
def test_policy_few_tokens(lens, reduction, kl, per_token):
    t = Tokens(sum(lens), lens, d=72)
    adv = np.random.default_rng(5).standard_normal(t.T if per_token else len(t.lens))
    check_policy(t, adv, kl, reduction=reduction)


@pytest.mark.parametrize("lens", [[5, 0, 31, 1, 100, 64], [128, 128], [0, 257], [4] * 64, [3] * 66])
@pytest.mark.parametrize("kind,smoothing", [(0, 0.15), (1, 0.0), (2, 0.0)])
@pytest.mark.parametrize("mean_tokens", [False, True])
def test_pref_few_tokens(lens, kind, smoothing, mean_tokens):
    check_pref(Tokens(sum(lens), lens, d=72), True, kind, mean_tokens, smoothing=smoothing)


@pytest.mark.parametrize("d", [8, 16, 248, 256, 264, 1024, 2056, 11008])
def test_row_widths_of_many_tokens(d):
    check_policy(Tokens(d, [7, 300], d=d), [1.0, -0.5], True)
    check_pref(Tokens(d + 1, [290, 30], d=d))


@pytest.mark.parametrize("off", [[0, 900, 600], [0, 300, 700], [5, 300, 600], [0, -4, 600]])
def test_offsets_out_of_order_among_many_tokens_are_reported(off):
    t = Tokens(9, [300, 300])
    t.doff = torch.tensor(off, dtype=torch.int32, device="cuda")
    pref(t, True, SIGMOID, True, 0.1, 0.0, 0.0, 1.0, status=lora.LORA_EINVAL)
    assert (t.dh[t.T:] == 55).all() and float(t.w[0]) == 55 and float(t.w[t.T + 1]) == 55


def test_rows_of_many_tokens_in_place():
    """dh over dh_nll: the same bits as apart, however far ahead rows are read."""
    t = Tokens(41, [3000, 2500], d=1032, junk=False)
    check_policy(t, [1.0, -0.5], True)
    t2 = Tokens(41, [3000, 2500], d=1032, junk=False)
    policy(t2, [1.0, -0.5], True, dh=t2.dh_nll)
    assert torch.equal(t2.dh_nll, t.dh[:t.T])


@pytest.mark.parametrize("lens", [[3, 4], [3, 400]])
@pytest.mark.parametrize("per_token", [False, True])
def test_policy_advantage_zero_with_a_ratio_beyond_fp32(lens, per_token):
    """0 * rho is 0 for every finite rho = exp(delta): exp(89) is 4e38."""
    t = Tokens(60, lens, masked=False, junk=False)
    t.nll[0], t.old[0] = 1.0, 90.0
    t.nll[1], t.old[1] = 0.5, 700.0
    for k in ("nll", "old"):
        t.dev[k] = f32(getattr(t, k))
    adv = np.where(np.arange(t.T) < 3, 0.0, 0.5) if per_token else [0.0, 0.5]
    for reduction in (SUM, MEAN_TOKENS, MEAN_SEQS):
        policy(t, adv, False, reduction=reduction, scale=1.3)
        loss, w, _, _ = oracle.policy_loss(t.nll, t.old, None, np.asarray(adv, np.float32), t.mask, t.off,
                                           float(np.float32(0.2)), 0.25, 0.0, float(np.float32(1.3)), reduction)
        assert w[0] == 0 and w[1] == 0 and math.isfinite(loss)
        assert np.allclose(t.w[1:-1].double().cpu().numpy(), w, rtol=2e-6, atol=0)
        # the terms left are A rho of one sign: their sum is the sum of their magnitudes
        assert float(t.loss[0]) == pytest.approx(loss, rel=2e-6)
        t.check_rows(w)


@pytest.mark.parametrize("lens", [[3, 4], [3, 400]])
@pytest.mark.parametrize("reduction", [SUM, MEAN_TOKENS, MEAN_SEQS])
def test_policy_beta_zero_with_a_divergence_beyond_fp32(lens, reduction):
    """beta 0 with a reference model, for the statistics alone: loss and weights are those without one, to the bit."""
    t = Tokens(61, lens, masked=False, junk=False)
    t.nll[0], t.old[0], t.ref[0] = 97.0, 97.0, 1.0
    for k in ("nll", "old", "ref"):
        t.dev[k] = f32(getattr(t, k))
    policy(t, [0.7, -0.5], False, beta=0.0, reduction=reduction)
    want = [v.clone() for v in (t.loss[:1], t.w, t.dh)]
    assert torch.isfinite(t.loss[0])
    stats = policy(t, [0.7, -0.5], True, beta=0.0, reduction=reduction)
    assert all(torch.equal(a, b) for a, b in zip(want, (t.loss[:1], t.w, t.dh)))
    assert stats[0] == math.inf  # exp(96) / 403 is 1e39


@pytest.mark.parametrize("lens", [[2, 1], [300, 1]])
@pytest.mark.parametrize("off", [-1, 0, 1])
def test_pref_hinge_beside_its_corner(lens, off):
    """m = 1 + off 2^-40, exact in the sums' pairs of fp32 and 1 in fp32: below 1 the loss has a slope."""
    t = Tokens(62, lens, d=16, masked=False, junk=False)
    t.nll[:] = 0.0
    t.ref[:] = 0.0
    t.ref[0], t.ref[1] = 1.0, off * 2.0 ** -40
    for k in ("nll", "ref"):
        t.dev[k] = f32(getattr(t, k))
    check_pref(t, kind=1, beta=1.0, margin=0.0, scale=1.0)
    assert float(t.w[1]) == (1.0 if off < 0 else 0.0)  # d loss / d nll of the preferred answer


@pytest.mark.parametrize("lens", [[40], [400, 3]])
@pytest.mark.parametrize("reduction", [MEAN_TOKENS, MEAN_SEQS])
def test_rows_whose_weight_rounds_to_zero(lens, reduction):
    """exp(-103) is fp32's smallest number; over 40 tokens and more it is a weight of zero, and its row is zeros."""
    t = Tokens(63, lens, masked=False, junk=False)
    t.nll[2], t.old[2] = 104.0, 1.0
    for k in ("nll", "old"):
        t.dev[k] = f32(getattr(t, k))
    t.dh_nll[2] = float("inf")
    policy(t, [1.0] * len(lens), False, reduction=reduction, scale=1.0)
    assert t.w[3] == 0 and (t.dh[2] == 0).all() and torch.isfinite(t.dh).all()


@pytest.mark.parametrize("lens", [[30, 40, 50, 7], [3000, 40, 900, 7]])
@pytest.mark.parametrize("which", ["policy", "pref"])
def test_in_a_graph(lens, which):
    """Captured once, replayed on other values in place."""
    t = Tokens(70, lens, d=72)
    adv = f32([0.5, -1.0, 2.0, 0.1])
    extra = torch.zeros(4, device="cuda")
    if which == "policy":
        args = lora.make_policy_args(t.T, 4, t.d, t.doff, t.dev["nll"], t.dev["old"], adv, t.loss, ref_nll=t.dev["ref"],
                                     mask=t.dmask, beta=0.05, reduction=MEAN_SEQS, stats=extra, **t.outputs())
        fn, size = lora.lora_policy_fwd_bwd, lora.lora_policy_workspace_size(args)
    else:
        args = lora.make_pref_args(t.T, 2, t.d, t.doff, t.dev["nll"], t.loss, ref_nll=t.dev["ref"], mask=t.dmask,
                                   rewards=extra, **t.outputs())
        fn, size = lora.lora_pref_fwd_bwd, lora.lora_pref_workspace_size(args)
    ws = G.workspace(size)
    fn(args, ws, ws.numel())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fn(args, ws, ws.numel())
    outs = [t.loss[:1], t.w[1:-1], t.dh[:t.T], extra]
    last = None
    for seed in (71, 72):
        other = Tokens(seed, lens, d=72)
        for k in ("nll", "old", "ref"):
            t.dev[k].copy_(other.dev[k])
        t.dmask.copy_(other.dmask)
        t.dh_nll.copy_(other.dh_nll)
        fn(args, ws, ws.numel())
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)) and torch.isfinite(want[0]).all()
        assert last is None or not torch.equal(last[0], want[0])
        last = want
    assert lora.lora_read_status() == lora.LORA_OK
