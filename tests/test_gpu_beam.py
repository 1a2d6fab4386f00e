"""A beam search's selection and reordering on the GPU against float64 definitions.

Beams and tokens are compared exactly.  Scores: one rounding to float32, u |s| with u = 2^-24, and the normaliser's error: what is summed in float32 lies below the
collecting threshold, each term with the relative error of an exponential whose argument (at most 2^20 in magnitude, and at most about 30 where it counts) is one rounded multiply-add,
(4 + 30) u, sums of n terms 8 sqrt(n) u: together less than 64 u for n up to 2^18 of the sum (8 sqrt(n) u bounds the few additions of one thread, n / 256, by far)."""
import math

import numpy as np
import pytest
import torch

import paper_2603_25011_amd as lsr
from oracle import beam_oracle as orc
from paper_2603_25011_amd import beam, binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return t.detach().double().cpu().numpy()


def check(X, scores, K, T=1.0, finished=None, end_id=0):
    got = beam.beam_select(X, scores, K, T, finished, end_id)
    want = orc.select(host(X), host(scores), K, T, None if finished is None else finished.cpu().numpy() != 0, end_id)
    assert got[0].shape == got[1].shape == got[2].shape == (X.shape[0], K)
    assert np.array_equal(got[1].cpu().numpy(), want[1]), "beams"
    assert np.array_equal(got[2].cpu().numpy(), want[2]), "tokens"
    with np.errstate(invalid="ignore", over="ignore"):
        s, w = host(got[0]), want[0].astype(np.float32).astype(np.float64)       # (what lies beyond float32 is an infinity there too)
        same = (s == w) | (np.isnan(s) & np.isnan(w))
        bad = ~(same | (np.abs(s - want[0]) <= U * np.abs(want[0]) + 64 * U))
    assert not bad.any(), f"scores: {bad.sum()} off, {s[bad][0]} for {want[0][bad][0]} at {np.argwhere(bad)[0]}"
    return got


def logits(gen, B, beams, V, dtype, pitch=None, hot=20):
    x = torch.randn(B, beams, pitch or V, generator=gen) * 1.5
    at = torch.randint(0, V, (B, beams, min(hot, V)), generator=gen)
    x.scatter_(2, at, torch.rand(at.shape, generator=gen) * 8 + 2)
    return x.to(TYPES[dtype]).to(DEV)[..., :V]


def scores_of(gen, B, beams):
    return -(torch.rand(B, beams, generator=gen) * 2).cumsum(1).to(DEV) - 3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,beams,V,K,pitch,T", [(1, 1, 1, 1, 1, 1.0), (2, 3, 5, 15, 5, 1.0), (1, 4, 30522, 8, 30522, 1.0), (3, 5, 1000, 10, 1001, 0.7), (2, 8, 4099, 16, 4100, 2.0),
                                                 (1, 64, 700, 128, 703, 1.0), (40, 2, 300, 3, 300, 1.0), (1, 2, 70001, 128, 70001, 0.5), (70, 16, 513, 32, 513, 1.0)])
def test_selection(B, beams, V, K, pitch, T, dtype):
    gen = torch.Generator().manual_seed(B + 10 * beams + V)
    check(logits(gen, B, beams, V, dtype, pitch), scores_of(gen, B, beams), K, T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_excluded_tokens_finished_beams_and_empty_places(dtype):
    gen = torch.Generator().manual_seed(1)
    x, s = logits(gen, 6, 4, 900, dtype), scores_of(gen, 6, 4)
    x[0, :, 3:] = -math.inf                    # three tokens each: twelve continuations for sixteen places
    x[1, 2] = -math.inf                        # a beam with none
    x[2] = -math.inf                           # a sequence with none
    s[3, 1:] = -math.inf                       # the first step
    s[4] = -math.inf
    fin = torch.zeros(6, 4, dtype=torch.bool, device=DEV)
    fin[5, 1:] = True
    fin[2, 3] = True
    got = check(x, s, 16, 1.0, fin, 7)
    assert (got[0][0, 12:] == -math.inf).all() and (got[2][0, 12:] == 7).all() and (got[1][3] == 0).all()
    check(x, s, 16, 1.0, fin.to(torch.int64) * 5, 7)
    check(x, s, 1, 1.0, fin, 0)
    fin[:] = True
    got = check(x, s, 5, 1.0, fin, 899)
    # the logits of finished beams and of beams of -inf are not read
    x[:] = math.nan
    again = check(x, s, 5, 1.0, fin, 899)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_hard_rows(V, dtype):
    gen = torch.Generator().manual_seed(V)
    lowest = torch.finfo(TYPES[dtype]).min
    x = logits(gen, 14, 2, V, dtype)
    s = scores_of(gen, 14, 2)
    x[0] = 1.25                                # all alike
    x[1, 0] = torch.arange(V, device=DEV).to(x.dtype)         # ascending: every batch beats the threshold
    x[2, 0] = -torch.arange(V, device=DEV).to(x.dtype)
    x[3] = lowest                              # a mask of the type's lowest value over everything
    x[4, :, :-1] = lowest                      # or all but one
    x[5, 1] = x[5, 0]                          # the same row twice
    s[5, 1] = s[5, 0]
    x[6, 0, V // 2] = math.nan
    x[7, 1, V - 1] = math.inf
    x[8, 0] = math.nan
    s[9, 0] = math.nan
    s[10, 1] = math.inf
    x[11] = x[11] * 1000                       # far apart
    x[12] = (x[12] > 2).to(x.dtype)            # two values only
    x[13] = x[13] * 1e-3 - 1e4                 # far from zero
    check(x, s, 16, 1.0, None, 3)
    check(x, s, 16, 0.05, None, 3)


def check_alike(X, scores, K):
    """Continuations of different beams may be equal in exact arithmetic while either side rounds them apart (score 1 with logits 1, 0, 1 and score 0 with 1, 1, 0: the
    second token of the one and the first of the other both have -log(2 + 1/e)).  A score of either beam is off by at most 64 u (its normaliser, see above) + u |s|, so two
    whose exact scores differ by less than 128 u + 2 u |s| may stand in either order: a place holds what is wanted there or another continuation that near it, none twice."""
    got = beam.beam_select(X, scores, K)
    x, s = host(X), host(scores)
    want = orc.select(x, s, K)
    values, beams, tokens = (t.cpu().numpy() for t in got)
    for b in range(X.shape[0]):
        seen = set()
        for k in range(K):
            w, m, t = want[0][b, k], int(beams[b, k]), int(tokens[b, k])
            assert (math.isnan(w) and math.isnan(values[b, k])) or w == values[b, k] or abs(w - values[b, k]) <= U * abs(w) + 64 * U
            if not math.isfinite(w):
                assert (m, t) == (want[1][b, k], want[2][b, k])
                continue
            assert (m, t) not in seen
            seen.add((m, t))
            if (m, t) != (want[1][b, k], want[2][b, k]):
                z = x[b, m]
                own = s[b, m] + ((z[t] - z.max()) - np.log(np.exp(z - z.max()).sum()))
                assert abs(own - w) <= 128 * U + 2 * U * abs(w), (b, k, own, w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,beams,V,K", [(2, 16, 30522, 32), (1, 64, 1500, 128), (3, 5, 20000, 7), (2, 12, 700, 1)])
def test_many_candidates_of_equal_score(B, beams, V, K, dtype):
    """More than are ranked against each other: by beam and token, whatever is alike."""
    gen = torch.Generator().manual_seed(V)
    x = torch.zeros(B, beams, V, dtype=TYPES[dtype], device=DEV)
    s = torch.zeros(B, beams, device=DEV)
    got = check(x, s, K)
    assert (got[1] == 0).all() and torch.equal(got[2], torch.arange(K, dtype=torch.int32, device=DEV).expand(B, K))
    s[:, 0] = -1.0                             # the best are another beam's
    check(x, s, K)
    x[:] = (torch.rand(B, beams, V, generator=gen) < 0.5).to(x)          # two values
    s[:] = torch.randint(0, 2, (B, beams), generator=gen).to(s)
    check_alike(x, s, K)
    x[0, beams // 2, V // 3] = math.nan        # a beam that comes first, and has places enough
    check_alike(x, s, K)
    x[:, :, 3:] = -math.inf                    # fewer than there are places for, and then none
    check_alike(x, s, K)
    x[:] = -math.inf
    check_alike(x, s, K)


def test_the_first_of_equal_beams_wins():
    x = torch.zeros(1, 3, 50, device=DEV)
    s = torch.zeros(1, 3, device=DEV)
    got = check(x, s, 60)
    assert got[1][0].tolist() == [0] * 50 + [1] * 10 and got[2][0].tolist() == list(range(50)) + list(range(10))


@pytest.mark.parametrize("T", [1e-30, 1e-6, 1e6, 1e30])
def test_extreme_temperatures(T):
    gen = torch.Generator().manual_seed(2)
    check(logits(gen, 2, 1, 3000, "f32"), scores_of(gen, 2, 1), 8, T)


def test_normaliser_is_closer_than_float32():
    """What reaches the threshold is summed in 64 bits: against float64 the scores are one rounding off."""
    gen = torch.Generator().manual_seed(3)
    x, s = logits(gen, 8, 4, 30522, "bf16", hot=32), torch.zeros(8, 4, device=DEV)
    for m in range(4):
        got = beam.beam_select(x[:, m:m + 1], s[:, m:m + 1], 1)[0]
        want = orc.select(host(x[:, m:m + 1]), host(s[:, m:m + 1]), 1)[0]
        # scores here are 1 to 4 in magnitude: half a step of float32 is 2^-23 at most; the sums' own error is a tenth of that
        assert np.abs(host(got) - want).max() <= 1.1 * 2.0 ** -23


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_beat_every_threshold(dtype):
    """Ascending logits, of one wave alone, or alike but for their index: more than the list holds in every batch.  Equal beams have equal sums, call after call."""
    gen = torch.Generator().manual_seed(31)
    V = 30011
    x = torch.zeros(5, 3, V, device=DEV)
    x[0] = torch.arange(V, device=DEV) * 3e-4
    x[1] = (torch.arange(V) * 1e-3 + torch.rand(V, generator=gen) * 0.01).to(DEV)
    x[2] = torch.where((torch.arange(V) // 512 % 4 == 1).to(DEV), x[1, 0] + 1.0, x[1, 0] - 40.0)
    x[3] = 2.0
    x[4] = (torch.arange(V, device=DEV) // 5000).float()
    x[3, :, V // 2:] = 3.0
    x = x.to(TYPES[dtype])
    s = torch.zeros(5, 3, device=DEV)
    got = check(x, s, 16)
    check(x, s, 128)
    check(x, s, 1)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(got, beam.beam_select(x, s, 16)))


def test_rows_beyond_4_gib():
    V = 1 << 26
    x = torch.full((2, 20, V), -1.0, dtype=torch.bfloat16, device=DEV)
    x[1, 19, V - 1] = 30.0
    x[1, 3, 5] = 29.0
    s = torch.zeros(2, 20, device=DEV)
    got = beam.beam_select(x, s, 3)
    assert got[1][1, :2].tolist() == [19, 3] and got[2][1, :2].tolist() == [V - 1, 5] and got[2][0].tolist() == [0, 1, 2]


def test_selection_repeats_its_bits_and_runs_in_a_graph():
    gen = torch.Generator().manual_seed(4)
    x, s = logits(gen, 5, 6, 9000, "bf16"), scores_of(gen, 5, 6)
    x[0] = 0.5
    first = beam.beam_select(x, s, 12)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, beam.beam_select(x, s, 12)))
    tokens = torch.randint(0, 9000, (5, 6, 11), generator=gen, dtype=torch.int32).to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        beam.beam_reorder(tokens, beam.beam_select(x, s, 6)[1])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = beam.beam_select(x, s, 6)
        moved = beam.beam_reorder(tokens, out[1])
    for k in range(4):
        x.copy_(logits(gen, 5, 6, 9000, "bf16"))
        s.copy_(scores_of(gen, 5, 6))
        torch.cuda.synchronize()
        graph.replay()
        want = beam.beam_select(x, s, 6)
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(moved, beam.beam_reorder(tokens, want[1]))


def test_refusals():
    x, s = torch.zeros(2, 3, 10, device=DEV), torch.zeros(2, 3, device=DEV)
    for bad in (lambda: beam.beam_select(x[0], s, 2), lambda: beam.beam_select(x, s[:, :2], 2), lambda: beam.beam_select(x, s, 2, finished=s[:1] > 0)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: beam.beam_select(x, s, 0), lambda: beam.beam_select(x, s, 31), lambda: beam.beam_select(x, s, 2, 0.0), lambda: beam.beam_select(x, s, 2, end_id=10)):
        with pytest.raises(lsr.LsrError):
            bad()
    with pytest.raises(TypeError):
        beam.beam_select(x.half(), s, 2)
    assert beam.beam_select(x[:0], s[:0], 2)[0].shape == (0, 2)


# ---- reordering ----

def parents_of(gen, B, beams, K):
    return torch.randint(0, beams, (B, K), generator=gen, dtype=torch.int32).to(DEV)


@pytest.mark.parametrize("B,beams,K", [(1, 1, 1), (3, 4, 4), (2, 5, 9), (7, 8, 1)])
def test_reorder(B, beams, K):
    gen = torch.Generator().manual_seed(B)

    def ints(*shape, dtype):
        return torch.randint(0, 100, shape, generator=gen).to(dtype).to(DEV)
    states = [ints(B, beams, dtype=torch.float32), ints(B, beams, 33, dtype=torch.int32), ints(B, beams, 3, dtype=torch.uint8), ints(B, beams, 7, dtype=torch.bfloat16),
              ints(B, beams, 12, 50, 64, dtype=torch.bfloat16)[:, :, :, :17], ints(B, beams, 1000, dtype=torch.float64), ints(beams, B, 40, dtype=torch.int64).transpose(0, 1),
              ints(B, 1, 24, dtype=torch.float32).expand(B, beams, 24), ints(B, beams, 6, 10, 8, dtype=torch.float32)[:, :, ::2, 1:5, ::2],
              ints(B, beams, 11, dtype=torch.int16)[..., 3:], torch.zeros(B, beams, 0, device=DEV), ints(B, beams, 2, 3, 4, dtype=torch.bool)]
    p = parents_of(gen, B, beams, K)
    got = beam.beam_reorder(states, p)
    for x, y in zip(states, got):
        assert y.dtype == x.dtype and y.is_contiguous()
        if x.dtype == torch.bfloat16:
            x, y = x.float(), y.float()
        assert np.array_equal(y.cpu().numpy(), orc.reorder(x.cpu().numpy(), p.cpu().numpy()))
    # into tensors of the program's own, caches of which only a part is in use among them
    big = [torch.full((B, K, 12, 60, 64), -1.0, dtype=torch.bfloat16, device=DEV), torch.full((B, K, 40), -1, dtype=torch.int32, device=DEV)]
    out = beam.beam_reorder([states[4], states[1]], p, [big[0][:, :, :, :17], big[1][..., 2:35]])
    assert torch.equal(out[0], got[4]) and torch.equal(out[1], got[1]) and (big[0][:, :, :, 17:] == -1).all()
    assert (big[1][..., :2] == -1).all() and (big[1][..., 35:] == -1).all()
    # one tensor, more tensors than a launch describes
    assert torch.equal(beam.beam_reorder(states[1], p), got[1])
    many = beam.beam_reorder([states[1]] * 70 + [states[5]], p)
    assert all(torch.equal(m, got[1]) for m in many[:70]) and torch.equal(many[70], got[5])


def test_reorder_parents_outside_the_beams_give_zeros():
    x = torch.randn(3, 4, 50, device=DEV)
    p = torch.tensor([[0, 4], [-1, 3], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device=DEV)
    assert np.array_equal(beam.beam_reorder(x, p).cpu().numpy(), orc.reorder(x.cpu().numpy(), p.cpu().numpy()))


def test_reorder_offsets_beyond_32_bits():
    x = torch.zeros(3, 2, 1 << 30, dtype=torch.uint8, device=DEV)
    x[2, 1, -1], x[2, 0, 5], x[0, 1, 1 << 29] = 9, 8, 7
    p = torch.tensor([[1, 1], [0, 0], [1, 0]], dtype=torch.int32, device=DEV)
    y = beam.beam_reorder(x, p)
    assert y[0, 0, 1 << 29] == y[0, 1, 1 << 29] == 7 and y[2, 0, -1] == 9 and y[2, 1, 5] == 8 and y.count_nonzero() == 4


def test_reorder_refusals():
    x, p = torch.zeros(2, 3, 10, device=DEV), torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    wide = torch.zeros(2, 3, 20, device=DEV)
    for bad in (lambda: beam.beam_reorder([x, x[:1]], p), lambda: beam.beam_reorder([x, x[:, :2]], p), lambda: beam.beam_reorder(x, p, torch.zeros(2, 3, 9, device=DEV)),
                lambda: beam.beam_reorder(x, p, x), lambda: beam.beam_reorder([x, x], p, [torch.zeros(2, 3, 10, device=DEV)]),
                lambda: beam.beam_reorder(x, p, torch.zeros(2, 1, 10, device=DEV).expand(2, 3, 10)),
                lambda: beam.beam_reorder(wide[..., :10], p, wide[..., 5:15]), lambda: beam.beam_reorder([x, x], p, [wide[..., :10], wide[..., :10]]),
                lambda: beam.beam_reorder(x, p, x.double()), lambda: beam.beam_reorder(x, p.long()), lambda: beam.beam_reorder(x[:, 0, 0], p)):
        with pytest.raises(ValueError):
            bad()
    assert beam.beam_reorder([], p) == []
    assert beam.beam_reorder(x[:0], p[:0]).shape == (0, 3, 10)


def test_reorder_out_that_holds_the_parents_and_views_of_other_signs():
    out = torch.zeros(2, 3, 2, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError, match="overlap"):
        beam.beam_reorder(torch.ones_like(out), out.view(-1)[:6].view(2, 3), out)
    x, p = torch.randn(2, 3, 5, dtype=torch.complex64, device=DEV), torch.tensor([[2, 0, 0], [1, 1, 2]], dtype=torch.int32, device=DEV)
    for y in (x.conj(), x.conj().imag):
        assert y.is_conj() or y.is_neg()
        want = torch.stack([y[b].resolve_conj().resolve_neg()[p[b].long()] for b in range(2)])
        assert torch.equal(beam.beam_reorder(y, p), want)
    with pytest.raises(ValueError, match="conjugated"):
        beam.beam_reorder(x, p, torch.zeros_like(x).conj())


def test_entry_points_are_the_package_own():
    assert lsr.lsr_beam_select is binding.lsr_beam_select and lsr.lsr_beam_reorder is binding.lsr_beam_reorder
