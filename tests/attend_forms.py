"""Problems that reach the forms of decode attention that few problems do: by what the call decides
(the expected form at 256 CUs, checked on the host) and what it has to compute (checked on a GPU)."""

# heads (q, kv, size), lengths, tokens of each request, whether causal; then the form: a workgroup per
# item or equal shares, KV heads side by side, waves of a workgroup, pieces of the longest request at least
FORMS = {
    # eight heads: a wave each, without a join of a workgroup's waves
    "a_wave_per_head": dict(heads=(8, 8, 64), lens=[14001, 700], tokens=[1, 1], causal=True,
                            direct=False, side=8, waves=8),
    "eight_waves_four_heads": dict(heads=(64, 8, 64), lens=[30011] * 4, tokens=[1, 2, 1, 1], causal=True,
                                   direct=False, side=4, waves=8),
    "a_wave_per_head_of_five_tokens": dict(heads=(8, 8, 64), lens=[36000, 17, 40001], tokens=[5, 0, 4], causal=True,
                                           direct=False, side=8, waves=8),
    "a_wave_per_head_of_forty_rows": dict(heads=(64, 8, 64), lens=[[300, 33, 64][i % 3] for i in range(140)],
                                          tokens=[[5, 1][i % 2] for i in range(140)], causal=True,
                                          direct=True, side=8, waves=8),
    # four waves, two and four heads side by side
    "four_waves_two_heads": dict(heads=(32, 4, 128), lens=[33001, 5, 60007, 47000], tokens=[5, 1, 3, 5], causal=True,
                                 direct=False, side=2, waves=4),
    "four_waves_four_heads": dict(heads=(32, 4, 128), lens=[33001] * 17, tokens=[5] + [1] * 16, causal=True,
                                  direct=False, side=4, waves=4),
    # one long request among short ones: more than 64 pieces joined by a wave a row
    "many_pieces_a_wave_a_row": dict(heads=(8, 1, 64), lens=[60000] + [64] * 20, tokens=[1] * 21, causal=True,
                                     direct=False, side=1, waves=8, pieces=200),
    "many_pieces_of_128": dict(heads=(4, 1, 128), lens=[33, 50000] + [90] * 18, tokens=[1, 2] + [1] * 18, causal=True,
                               direct=False, side=1, waves=8, pieces=150),
    # short requests, some of them empty, several heads to a workgroup
    "empty_items_two_heads": dict(heads=(8, 2, 64), lens=[[70, 0, 33][i % 3] for i in range(300)],
                                  tokens=[1 + (i % 4 == 1) for i in range(300)], causal=False,
                                  direct=True, side=2, waves=8),
    "empty_items_eight_heads": dict(heads=(16, 8, 64), lens=[[40, 129, 0, 1][i % 4] for i in range(140)],
                                    tokens=[i % 3 for i in range(140)], causal=False, direct=True, side=8, waves=8),
    "empty_items_four_heads_four_waves": dict(heads=(132, 4, 128), lens=[[50, 0][i % 2] for i in range(160)],
                                              tokens=[1] * 160, causal=False, direct=True, side=4, waves=4),
}
