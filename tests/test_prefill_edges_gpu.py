"""attn_paged_prefill and attn_paged_prefix_decode at the edges of what their arguments may hold."""
import math

import pytest
import torch

from paper_2506_12355_b200 import api
from test_paged_gpu import make_cache
from test_prefill_gpu import check_prefill, check_prefix, make_shared, run_prefill, wide
from test_rope_gpu import DT

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,new,length", [(300, 60, 70), (2, 300, 2000), (1, 40, 5000)])       # whole lists; cut ones, of two tiles and of one
def test_a_visible_key_that_is_no_number_shows_in_o_and_lse(kind, D, n, new, length):
    """A NaN in one K row of one K/V head: NaN in O and LSE of the rows that see it, whether one CTA has their list to itself or several;
    all other rows as if it were not there."""
    H, Hkv, page, dt = 4, 2, 16, DT[kind]
    kc, vc, tab, ks, vs = make_cache([length] * n, Hkv, D, page, dt, "head", 41)
    j = length - new // 2
    kc[tab[:, j // page].long().cuda(), 1, j % page, 3] = math.nan
    q = torch.randn(n * new, H, D, generator=torch.Generator().manual_seed(42)).to(dt).cuda()
    cu = i32([new * b for b in range(n + 1)])
    o, lse = api.attn_paged_prefill(q, kc, vc, tab.cuda(), i32([length] * n), cu, D ** -0.5)
    assert api.attn_last_device_status() == 0
    o, lse = o.view(n, new, H, D), lse.view(n, new, H)
    first = j - (length - new)                        # token that sees the key first
    assert torch.isnan(o[:, first:, 2:]).all() and torch.isnan(lse[:, first:, 2:]).all()
    for b in range(0, n, 50):
        rows = q.view(n, new, H, D)[b]
        check_prefill(o[b, :, :2], lse[b, :, :2], rows[:, :2], ks[b][:, :1], vs[b][:, :1], D ** -0.5, dt)
        check_prefill(o[b, :first], lse[b, :first], rows[:first], ks[b][:j], vs[b][:j], D ** -0.5, dt)


@pytest.mark.parametrize("n", [5, 90])
def test_a_common_key_that_is_no_number_shows_in_o_and_lse(n):
    D, H, Hkv, page, dt, lens = 128, 8, 2, 16, torch.bfloat16, [300 + b % 7 for b in range(n)]
    kc, vc, tab, ks, vs = make_shared(lens, [0, n], [280], Hkv, D, page, dt, "head", 43)
    kc[int(tab[0, 3]), 1, 5, 7] = math.nan
    q = torch.randn(n, H, D, generator=torch.Generator().manual_seed(44)).to(dt).cuda()
    o, lse = api.attn_paged_prefix_decode(q, kc, vc, wide(tab, page, Hkv, D).cuda(), i32(lens), i32([0, n]), i32([280]), D ** -0.5)
    assert api.attn_last_device_status() == 0
    assert torch.isnan(o[:, 4:]).all() and torch.isnan(lse[:, 4:]).all()
    for b in range(n):
        check_prefill(o[b:b + 1, :4], lse[b:b + 1, :4], q[b:b + 1, :4], ks[b][:, :1], vs[b][:, :1], D ** -0.5, dt)


def malformed(lens, tokens, cu, seed=45):
    """One call over 3 sequences whose lists are not what they should be: (o, lse, q, keys, values, status), rows preset to 7."""
    D, H, Hkv, page, dt = 64, 4, 2, 16, torch.float16
    kc, vc, tab, ks, vs = make_cache(lens, Hkv, D, page, dt, "head", seed)
    q = torch.randn(tokens, H, D, generator=torch.Generator().manual_seed(seed + 1)).to(dt).cuda()
    o, lse = torch.full_like(q, 7.0), torch.full((tokens, H), 7.0, device="cuda")
    api.attn_paged_prefill(q, kc, vc, tab.cuda(), i32(lens), i32(cu), 0.125, o, lse)
    return o, lse, q, ks, vs, api.attn_last_device_status()


def check_rows_of(case, first, end, b, last):
    """Token first sees the keys 0 .. last of sequence b, the next one key more, and so on."""
    o, lse, q, ks, vs, _ = case
    n = last + end - first                           # keys behind the last token: none
    check_prefill(o[first:end], lse[first:end], q[first:end], ks[b][:n], vs[b][:n], 0.125, torch.float16)


def test_lists_that_reach_beyond_the_tokens_are_cut_and_reported():
    lens = [200, 64, 40]
    case = malformed(lens, 60, [0, 20, 40, 60])
    assert case[5] == 0
    check_rows_of(case, 40, 60, 2, 20)
    case = malformed(lens, 50, [0, 20, 40, 60])               # the last sequence's new tokens are 10 then
    assert case[5] == 13
    check_rows_of(case, 0, 20, 0, 180)
    check_rows_of(case, 20, 40, 1, 44)
    check_rows_of(case, 40, 50, 2, 30)
    case = malformed(lens, 60, [-4, 20, 40, 60])
    assert case[5] == 13
    check_rows_of(case, 0, 20, 0, 180)
    check_rows_of(case, 40, 60, 2, 20)
    case = malformed([200, 64, 0], 50, [0, 20, 40, 60])       # a padded sequence's list does not matter
    assert case[5] == 0 and (case[0][40:] == 7).all() and (case[1][40:] == 7).all()


def test_lists_that_run_backwards():
    lens = [200, 64, 40]
    case = malformed(lens, 60, [0, 40, 20, 60])               # tokens 20 .. 39 are in two lists
    check_rows_of(case, 0, 20, 0, 160)
    check_rows_of(case, 40, 60, 2, 20)
    case = malformed(lens, 70, [50, 10, 10, 30])              # the last sequence has tokens 10 .. 29
    check_rows_of(case, 10, 30, 2, 20)
    for rows in (slice(0, 10), slice(30, 70)):
        assert (case[0][rows] == 7).all() and (case[1][rows] == 7).all()
    case = malformed(lens, 60, [50, 10, 10, 10])
    assert case[5] == 0 and (case[0] == 7).all() and (case[1] == 7).all()
    case = malformed(lens, 60, [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, -2 ** 31])     # sequence 1 has all tokens
    assert case[5] == 13
    check_rows_of(case, 0, 60, 1, 4)


@pytest.mark.parametrize("starts,prefix", [([0, 3, 1], [160, 160]), ([-5, 2, 99], [160, 160]), ([3, 0, 3], [-1, 2 ** 31 - 1]), ([7, 9], [5]), ([0, 3], [-1]),
                                           ([-2 ** 31, 2 ** 31 - 1], [160])])
def test_groups_that_run_backwards_or_past_the_batch(starts, prefix):
    """Each sequence is in a group whose common keys are its own, or in none: the results are those of plain decoding."""
    D, H, Hkv, page, dt, lens = 64, 4, 2, 16, torch.float16, [200, 300, 250]
    kc, vc, tab, ks, vs = make_shared(lens, [0, 3], [160], Hkv, D, page, dt, "head", 9)
    q = torch.randn(3, H, D, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    o, lse = api.attn_paged_prefix_decode(q, kc, vc, wide(tab, page, Hkv, D).cuda(), i32(lens), i32(starts), i32(prefix), 0.125)
    assert api.attn_last_device_status() == 0
    check_prefix(o, lse, q, ks, vs, 0.125, dt)


@pytest.mark.parametrize("D,kind", [(64, "bf16"), (128, "fp16")])
def test_prefill_of_many_sequences_most_of_which_bring_little(D, kind):
    """More sequences than one lane's share of the plan fits into a few rounds: most bring no token or one, some are padding, a run of 900
    brings nothing at all."""
    lens, news = [], []
    for b in range(2500):
        if 800 <= b < 1700:
            lens.append(3 if b % 2 else 0)
            news.append(0)
        else:
            lens.append(0 if b % 11 == 3 else 1 + (b * 7) % 50)
            news.append(0 if lens[-1] == 0 or b % 5 == 1 else (lens[-1] if b % 97 == 0 else 1))
    run_prefill(lens, news, 4, 2, D, 16, kind, "head", seed=46)
