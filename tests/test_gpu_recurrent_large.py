"""The recurrent block's operators at sizes that reach the kernel forms of large launches, against the CPU oracle, every residue equal.

An inner product takes the division inside from 768 slices on (limbs that stay x items of a batch x blocks of 2^11 points): of the three forms that such an inner product has here the
sizes below give launches on both sides of that count, with the slices in brackets.  A product with a rotated operand and the gates' gradient take batches of eight at most, sums that are
relinearised batches of sixteen; two streams halve them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2604_16834_amd as hx  # noqa: E402
from test_gpu_recurrent import Turns, ciphertexts, equal, grad_case, leave_nothing, norm_case, place, random_key, scan_case, world  # noqa: E402, F401


# ------------------------------------------------------------------------------------------ products with a rotated operand
def step_case(ring, level, channels, heads, k, seed, strided=False):
    rng = np.random.default_rng(seed)
    turns = Turns(ring, rng)
    p, orc = turns.p, turns.orc
    gate, state, x = (ciphertexts(rng, p, level, n) for n in (heads, channels, channels))
    (rot, cross), dev = turns(-1)
    per = channels // heads
    got = hx.he_scan_step(turns.ctx, level, place(gate, strided), place(state, strided), dev[1], dev[0], x=place(x, not strided) if k else None, k=k or 0)
    equal(got, [orc.turned_product(gate[c // per], state[c], level, -1, rot, cross, k or 0, x[c] if k else None) for c in range(channels)])


@pytest.mark.parametrize("k", [3 << 49, None])
@pytest.mark.parametrize("ring,level,channels,heads", [((14, 14, 5, 3, 50), 13, 16, 4),   # two streams, eight each (832)
                                                       ((14, 14, 5, 3, 50), 12, 8, 8),    # (768)
                                                       ((14, 14, 5, 3, 50), 12, 7, 1),    # (672)
                                                       ((13, 26, 9, 3, 50), 25, 8, 2),    # (800)
                                                       ((16, 7, 3, 3, 50), 6, 5, 1),      # (960)
                                                       ((16, 7, 3, 3, 50), 6, 7, 7)])     # two streams, four and three (768, 576)
def test_steps_of_many_slices(ring, level, channels, heads, k):
    step_case(ring, level, channels, heads, k, channels + level, strided=heads == 1)


@pytest.mark.parametrize("channels,heads,steps,reverse", [(14, 2, 3, False),   # batches of eight, the last step's of seven (832, 768, 616)
                                                         (8, 8, 1, True),      # two streams (416), then the gradient of all eight gates (768)
                                                         (7, 7, 1, False)])    # likewise, of seven (672)
def test_scans_and_gradients_of_many_slices(channels, heads, steps, reverse):
    scan_case((14, 14, 5, 3, 50), 13, channels, heads, steps, reverse, channels, strided=reverse)


def test_scan_and_gradients_of_the_largest_ring():
    """N = 2^17: five rows in a batch (960), the last step without gates (512)."""
    scan_case((17, 4, 2, 2, 50), 3, 4, 1, 2, False, 17)


# ------------------------------------------------------------------------------------------ relinearised sums
@pytest.mark.parametrize("level,channels,affine", [(15, 17, False),   # two streams, nine and eight (936, 832)
                                                   (15, 14, False),   # two streams, seven each (728)
                                                   (15, 17, True)])   # a level less (864, 768)
def test_gradients_of_a_norm_of_many_slices(level, channels, affine):
    grad_case((14, 16, 6, 3, 50), level, channels, affine, [], channels + affine, strided=affine, want_gain=False, want_bias=False)


def test_gradients_of_a_norm_of_a_large_ring():
    """N = 2^16, two streams, four channels each (768)."""
    grad_case((16, 9, 3, 3, 50), 8, 8, False, [(1,)], 8, want_gain=False)


@pytest.mark.parametrize("level", [23, 24])
def test_a_single_relinearised_sum_of_many_slices(level):
    """N = 2^16: the layer norm's and the root-mean-square norm's sum of squares, one item (736, 768)."""
    ring = (16, 25, 9, 3, 50)
    norm_case(ring, level, 2, 0, False, False, level)
    rng = np.random.default_rng(level)
    p, orc, ctx = world(*ring)
    x, key = ciphertexts(rng, p, level, 2), random_key(rng, p)
    k = [int(rng.integers(-(1 << 62), 1 << 62)) for _ in range(3)]
    got = hx.he_norm_gate(ctx, level, hx.from_host(x), *k, (), hx.ckks_key_load(ctx, hx.from_host(key), 0))
    equal(got, orc.norm_gate(x, level, *k, (), key))


def test_layer_norm_and_its_gradients_of_the_largest_ring():
    norm_case((17, 5, 2, 3, 50), 4, 3, 0, True, True, 17)
    grad_case((17, 5, 2, 3, 50), 4, 2, True, [(1, 2, 3), (4,)], 18)


# ------------------------------------------------------------------------------------------ sums over slots
# A thread of the sums' kernel takes 8 (up to two digits) or 4 ciphertexts, halved while a half holds all or the launch has fewer than 1024 workgroups: N / 256 x limbs of the extended basis x groups
# of ciphertexts.  Every (digits, ciphertexts a thread) there is, by (ring, level, channels, both gradients or one): the sums run a level below, on channels or twice as many ciphertexts.
SUMS = {
    (1, 8): ((14, 5, 5, 1, 50), 4, 5, True),      # ten ciphertexts: eight and two
    (1, 4): ((14, 5, 5, 1, 50), 4, 3, True),      # four and two
    (1, 2): ((14, 5, 5, 1, 50), 4, 3, False),     # two and one
    (1, 1): ((14, 5, 5, 1, 50), 4, 1, False),
    (2, 8): ((14, 6, 3, 2, 50), 5, 5, True),
    (2, 4): ((14, 6, 3, 2, 50), 5, 3, True),
    (2, 2): ((14, 6, 3, 2, 50), 5, 3, False),
    (2, 1): ((14, 6, 3, 2, 50), 5, 1, False),
    (3, 4): ((14, 8, 3, 3, 50), 7, 3, True),
    (3, 2): ((14, 8, 3, 3, 50), 7, 3, False),
    (3, 1): ((14, 8, 3, 3, 50), 7, 1, False),
    (4, 4): ((14, 8, 2, 4, 50), 7, 3, True),
    (4, 2): ((14, 8, 2, 4, 50), 7, 3, False),
    (4, 1): ((14, 8, 2, 4, 50), 7, 1, False),
}


def ciphertexts_a_thread(log_n, limbs, digits, n):
    per = 8 if digits <= 2 else 4
    while per > 1 and (per // 2 >= n or (1 << log_n) // 256 * limbs * -(-n // per) < 1024):
        per //= 2
    return per


@pytest.mark.parametrize("form", list(SUMS))
def test_sums_over_slots_in_every_form(form):
    """A stage of seven rotations (several chains of additions), and one of two, the first of which reads what the stage before has written."""
    ring, level, channels, both = SUMS[form]
    log_n, num_q, num_p, dnum, _ = ring
    digits = -(-level // -(-num_q // dnum))  # level limbs a level below
    assert (digits, ciphertexts_a_thread(log_n, level + num_p, digits, channels * (1 + both))) == form
    grad_case(ring, level, channels, False, [(1, 2, 3, 4, 5, 6, 7), (8, -3)], 10 * digits + channels, want_gain=both)


@pytest.mark.parametrize("form", [(1, 8), (2, 8), (3, 4), (4, 2)])
def test_sums_over_slots_of_more_rotations_than_a_launch_holds(form):
    """35 rotations: a second launch adds to the first one's sums."""
    ring, level, channels, both = SUMS[form]
    grad_case(ring, level, channels, False, [tuple(range(1, 36))], channels, want_gain=both)


@pytest.mark.parametrize("channels", [8, 7])
def test_sums_over_slots_of_a_full_batch(channels):
    """Sixteen ciphertexts, eight a thread; fourteen, eight and six."""
    grad_case((14, 6, 3, 2, 50), 5, channels, False, [(1, 2, 3)], channels)
