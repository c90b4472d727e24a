"""How much memory the experts' calls ask for."""
import pytest

import paper_2511_11446_amd as ql


@pytest.mark.parametrize("T, k, E, K, I, N", [(16384, 8, 64, 2048, 1024, 2048), (4096, 2, 8, 2048, 1024, 2048), (2048, 8, 256, 7168, 2048, 7168), (500, 1, 1, 256, 4096, 256)])
def test_many_rows_ask_for_what_they_use(T, k, E, K, I, N):
    """Codes and scales of the tokens and of the gated products, outputs in binary16 with a byte for 64 of them, the plan; beside them no more than fp32 of the most rows
    that count as few (384 of one expert, else 12 of each of E or of 44)."""
    P, few, blocks = T * k, 384 if E == 1 else 12 * max(E, 44), lambda n: -(-n // 128)
    used = T * (K + 4 * blocks(K)) + P * (I + 4 * blocks(I)) + P * (2 * N + -(-N // 64)) + 8 * P + 8 * (P // 16 + min(P, E)) + 4 * E * (2 + P // 2048)
    assert used <= ql.experts_f8_workspace_bytes(T, k, E, K, I, N) <= used + 4 * few * (I + N) + 16 * 256


@pytest.mark.parametrize("E", [1, 2, 8, 44, 45, 64, 512])
def test_it_is_enough_for_every_call_of_fewer_rows(E):
    """On both sides of where rows stop being few and tiles change."""
    few = 384 if E == 1 else 12 * max(E, 44)
    for k in (1, 3):
        sizes = [ql.experts_f8_workspace_bytes(T, k, E, 256, 1024, 136) for T in sorted({1, 16, 17, few // (2 * k), few // k - 1, few // k, few // k + 1, 2 * few // k, 384 * E // k, 384 * E // k + 1, 400 * E})]
        assert sizes == sorted(sizes)
        assert all(ql.experts_f8_workspace_bytes(few // j, j, E, 256, 1024, 136) <= ql.experts_f8_workspace_bytes(few, j, E, 256, 1024, 136) for j in (1, 2, 3))
