"""The selective scan at the borders of what its coefficients and cuts allow: infinite and growing decays, every mapping of
workgroups to sequences, against the definition in 64 bits (sequence_reference) or exact whole numbers."""
import pytest
import torch

import sequence_reference as ref
from paper_1907_02129_amd import binding as icv

pytestmark = pytest.mark.gpu
# icv_scan_params::softplus above its public value: four, two or one states a lane, whole sequences or pieces of 64 rows
CUTS = {"auto": 0, "four": 1, "two": 2, "one": 3, "four_pieces": 1 | 1 << 2, "two_pieces": 2 | 1 << 2, "one_pieces": 3 | 1 << 2}


def ints(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")


def scan(x, dt, A, B, C, state, count, start=None, source=None, target=None, softplus=False, hook=0):
    """One call on dense float tensors: the output, the state slots and the workspace's size."""
    n, channels = x.shape
    seq = icv.make_sequences(count, n, ints(start), None, ints(source), ints(target))
    p = icv.make_scan_params(channels, A.shape[1], "f32", B.shape[1] // A.shape[1], softplus, state_slots=len(state))
    p.softplus |= hook << 8
    space = icv.selective_scan_workspace_bytes(p, seq)
    ws = torch.full((space // 4,), float("nan"), device="cuda") if space else None
    st, out = state.cuda(), torch.zeros(n, channels, device="cuda")
    icv.selective_scan(p, seq, x.cuda(), dt.cuda(), A.cuda(), B.cuda(), C.cuda(), None, None, None, st, out, ws)
    torch.cuda.synchronize()
    return out.cpu(), st.cpu(), space


@pytest.mark.parametrize("cut", [*CUTS, "step"])
@pytest.mark.parametrize("states", [16, 13])
@pytest.mark.parametrize("softplus", [False, True])
def test_infinite_coefficients_keep_the_state_over_steps_of_zero(cut, states, softplus):
    """A step of 0 keeps the state whatever its coefficient, any other step with a coefficient of -infinity or the lowest
    value forgets it.  Steps of 0 and 64 (which log(1 + exp(.)) leaves as it is) and small whole numbers make every state and
    output a whole number below 2^24, so that they have to be met exactly."""
    g = torch.Generator().manual_seed(states)
    n, ch = (9, 20) if cut == "step" else (300, 20)
    count = n if cut == "step" else 2
    whole = lambda *shape: torch.randint(-3, 4, shape, generator=g).float()  # noqa: E731
    x, B, C = whole(n, ch), whole(n, states), whole(n, states)
    delta = 64.0 * (torch.rand(n, ch, generator=g) < 0.2)
    delta[:, 1] = 0                              # whole pieces of steps of 0
    delta[60:200, 2] = 0
    delta[:, ch - 1] = 0
    dt = torch.where(delta > 0, delta, torch.full((), -200.0)) if softplus else delta
    A = torch.full((ch, states), -float("inf"))
    A[::3], A[:, 5] = -torch.finfo(torch.float32).max, -float("inf")
    A[ch - 1] = float("inf")                     # of steps of 0 alone
    state = whole(count, ch, states)
    slots = list(range(count))
    start = None if cut == "step" else [0, 170, 300]
    out, st, space = scan(x, dt, A, B, C, state, count, start, slots, slots, softplus, 0 if cut == "step" else CUTS[cut])
    assert cut == "auto" or (space > 0) == cut.endswith("pieces")
    want, want_state = torch.zeros(n, ch, dtype=torch.float64), state.double().clone()
    for i in range(count):
        for t in range(i, i + 1) if start is None else range(start[i], start[i + 1]):
            new = (delta[t] * x[t]).double()[:, None] * B[t].double()
            want_state[i] = torch.where(delta[t][:, None] > 0, new, want_state[i])
            want[t] = (want_state[i] * C[t].double()).sum(1)
    assert want.abs().max() < 2 ** 24 and want_state.abs().max() < 2 ** 24
    assert torch.equal(st.double(), want_state)
    assert torch.equal(out.double(), want)
@pytest.mark.parametrize("cut", [c for c in CUTS if c != "auto"] + ["four_128", "one_128"])
def test_decays_over_a_piece_past_the_range_of_float(cut):
    """Growing states (positive coefficients) whose growth over a piece is past 2^128, though no state ever is: states of zeros stay
    zeros, tiny ones grow to ordinary ones; and states that fall by more than 2^-128 over a piece and grow again."""
    n, ch, N = 256 + 20, 12, 8
    g = torch.Generator().manual_seed(3)
    hook = {"four_128": 1 | 2 << 2, "one_128": 3 | 2 << 2}.get(cut) or CUTS[cut]
    x, B, C = torch.zeros(n, ch), torch.rand(n, N, generator=g) + 0.5, torch.rand(n, N, generator=g) + 0.5
    dt, A, state = torch.ones(n, ch), torch.zeros(ch, N), torch.zeros(2, ch, N)
    # channels 0..3: 2^260 or more over 128 rows, nothing there until the last 20 rows
    A[:4] = torch.rand(4, N, generator=g) + 1.5
    x[256:, :4] = torch.randn(20, 4, generator=g)
    # channels 4..7: from 2^-120 or so by 2^2.1 a row for 90 rows
    A[4:8] = 1.46
    state[0, 4:8] = torch.exp2(-120 + torch.rand(4, N, generator=g))
    dt[90:, 4:8] = 0
    # channels 8..11: steps of -1 in the first 64 rows, then of +1: down by 2^-130 and up again (no state falls below 2^-126)
    A[8:] = 1.41
    dt[:64, 8:], dt[128:, 8:] = -1, 0
    state[0, 8:] = 2.0 ** 8 * (1 + torch.rand(4, N, generator=g))
    out, st, space = scan(x, dt, A, B, C, state, 1, [0, n], [0], [1], False, hook)
    assert (space > 0) == (hook >> 2 > 0)
    want, bound, st_want, sbound = ref.selective_scan(x, dt, A, B, C, None, None, None, state, [(0, n)], [0], [1], 1, False, torch.zeros(n, ch),
                                                      torch.float32, n if space else 0)
    assert want.isfinite().all() and bound.isfinite().all()
    ref.check("out", out, want, bound)
    ref.check("state", st, st_want, sbound)


@pytest.mark.parametrize("step", [True, False])
def test_activations_over_their_whole_range(step):
    """log(1 + exp(v)) (the state after one row from zeros), v / (1 + exp(-v)) as the scan's gate and as the convolution's
    activation, from -200 to 200 and next to 0, where results under 2^-126 and 2^-119 may be 0."""
    v = torch.cat([torch.linspace(-200, 200, 3201), torch.exp2(torch.arange(-126.0, 1)), -torch.exp2(torch.arange(-126.0, 1))])
    ch = len(v)
    one, z = torch.ones(1, ch), v[None]
    A, B, zeros = torch.zeros(ch, 1), torch.ones(1, 1), torch.zeros(1, ch, 1)
    p = icv.make_scan_params(ch, 1, "f32", state_slots=1)
    st, out = zeros.cuda(), torch.zeros(1, ch, device="cuda")
    seq = icv.make_sequences(1, 1, None if step else ints([0, 1]))
    assert icv.selective_scan_workspace_bytes(p, seq) == 0
    icv.selective_scan(p, seq, one.cuda(), z.cuda(), A.cuda(), B.cuda(), B.cuda(), None, None, None, st, out)
    want, bound, st_want, sbound = ref.selective_scan(one, z, A, B, B, None, None, None, zeros, [(0, 1)], [0], [0], 1, True, torch.zeros(1, ch),
                                                      torch.float32)
    ref.check("state", st, st_want, sbound + 2.0 ** -126)
    ref.check("out", out, want, bound + 2.0 ** -126)
    p = icv.make_scan_params(ch, 1, "f32", softplus=False)
    icv.selective_scan(p, seq, one.cuda(), one.cuda(), A.cuda(), B.cuda(), B.cuda(), None, z.cuda(), None, None, out)
    want, bound, _, _ = ref.selective_scan(one, one, A, B, B, None, z, None, zeros, [(0, 1)], [-1], [-1], 1, False, torch.zeros(1, ch), torch.float32)
    ref.check("gate", out, want, bound + 2.0 ** -119)
    filt = torch.ones(ch, 1)
    icv.causal_conv1d(icv.make_causal_conv_params(ch, 1, "f32"), seq, z.cuda(), filt.cuda(), None, None, out)
    want, bound, _ = ref.causal_conv(z, filt, None, torch.zeros(1, 0, ch), [(0, 1)], [-1], [-1], True, torch.zeros(1, ch), torch.float32)
    ref.check("activation", out, want, bound + 2.0 ** -119)
