"""The oracle of penalties / biases / masks and of the token counts against hand-worked cases and plain numpy."""
import numpy as np

import oracle


def test_hand_worked_rows():
    x = np.array([[2.0, -2.0, 1.0, 0.5, 4.0]] * 3, np.float32)
    counts = np.array([[0, 1, -32768, -32766, 0, 0, 0, 0]], np.int16)      # token 1 once, 2 in the prompt, 3 both (twice)
    out, _ = oracle.logits_adjust(x, [2], [0, 3], [0, 2], draft_tokens=[4, 1], counts=counts, repetition=[2.0], frequency=[0.25], presence=[0.5],
                                  bias_tokens=[[0, 4, 0]], bias_values=[[9.0, 10.0, -1.0]], n_bias=[3], mask=np.array([[0b11111], [0b11111], [0b10111]], np.uint32))
    np.testing.assert_allclose(out[0], [1.0, -4.75, 0.5, 0.25 - 0.5 - 0.5, 14.0])
    np.testing.assert_allclose(out[1], [1.0, -4.75, 0.5, -0.75, 2.0 - 0.75 + 10.0])     # draft 4 is in the history now
    np.testing.assert_allclose(out[2], [1.0, -5.0, 0.5, -np.inf, 11.25])                # and draft 1


def test_target_rows_equal_token_by_token_decoding():
    """Row i of a block is the draft-side row of a sequence whose counts already hold the drafts in front of it."""
    rng = np.random.default_rng(0)
    V, g = 50, 6
    x = rng.standard_normal((g + 1, V)).astype(np.float32)
    counts = rng.integers(0, 3, (1, 56)).astype(np.int16)
    drafts = rng.integers(0, 8, g)                                                      # repeats among them
    pen = dict(repetition=[1.3], frequency=[0.2], presence=[0.4])
    block, _ = oracle.logits_adjust(x, [g], [0, g + 1], [0, g], draft_tokens=drafts, counts=counts, **pen)
    for i in range(g + 1):
        c = oracle.token_counts_update(counts, V, drafts[:i], [0], [i])
        one, _ = oracle.logits_adjust(x[i:i + 1], cu_d=[0, 0], n_drafted=[0], draft_tokens=[0], counts=c, **pen)
        np.testing.assert_array_equal(block[i], one[0])


def test_counts():
    c = np.zeros((2, 8), np.int16)
    c[0, 3] = 32766
    c = oracle.token_counts_update(c, 7, [3, 3, 3, 9, -1, 5, 5], [0, 5], [5, 2])
    assert c.tolist() == [[0, 0, 0, 32767, 0, 0, 0, 0], [0, 0, 0, 0, 0, 2, 0, 0]]
    c = oracle.token_counts_update(c, 7, [3, 6, 5], [0, 2], [2, 1], prompt=True)
    assert c[0, 3] == -1 and c[0, 6] == -32768 and c[1, 5] == -32766                    # the mark leaves the count alone
    c = oracle.token_counts_update(c, 7, [0], [0, 0], [1, 0], reset=[1, 0])
    assert c[0].tolist() == [1, 0, 0, 0, 0, 0, 0, 0] and c[1, 5] == -32766
