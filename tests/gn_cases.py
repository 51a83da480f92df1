"""Group-norm shapes (n, hw, c, groups) that reach the kernels which the shapes of
test_gpu_gn.py leave out; tests/test_gn_launches.py checks that together they
launch every kernel that is compiled.  Names say what a shape is there for:
team_columns_vectors, a team being a workgroup (wg) or a wavefront (wave),
columns full (whole groups fill a power of two of them), padded or wide (more
than 64), vectors what a thread keeps at most, of eight channels or (s) one."""

RANGES = {
    "wg_full_1_one_channel_groups": (1, 1, 8, 8),
    "wg_padded_1": (1, 1, 24, 1),
    "wg_padded_1_sixes": (1, 1, 24, 6),
    "wg_wide_1": (1, 1, 520, 1),
    "wg_wide_1_halves": (1, 1, 520, 2),
    "wg_wide_2": (1, 2, 520, 1),
    "wg_wide_2_halves": (1, 2, 520, 2),
    "wg_padded_4_backward": (1, 17, 264, 1),
    "wg_padded_8_backward": (1, 33, 264, 1),
    "wg_padded_8_backward_quarters": (1, 33, 264, 4),
    "wg_wide_4_backward": (1, 3, 2056, 1),
    "wg_wide_4_backward_halves": (1, 3, 2056, 2),
    "wg_wide_8_backward": (1, 5, 2760, 4),
    "wg_wide_8": (1, 9, 2744, 1),
    "wg_wide_8_split_backward": (1, 9, 2792, 8),
    "wg_full_4_backward": (1, 1025, 8, 1),
    "wg_full_4_backward_fours": (1, 1025, 8, 2),
    "wg_full_8_backward": (1, 2049, 8, 1),
    "wave_full_1_one_channel_groups": (1024, 1, 8, 8),
    "wave_padded_1": (1030, 1, 24, 2),
    "wave_padded_2": (1029, 9, 40, 1),
    "wave_padded_2_fours": (1039, 9, 40, 4),
    "wave_full_2": (1032, 33, 16, 1),
    "wave_full_2_fours": (574, 9, 72, 18),
    "wave_full_2_wide_tile": (2048, 16, 64, 16),
    "split_wide": (1, 37, 888, 2),
    "split_wide_merged": (1, 266, 1048, 8),
    "split_padded_merged": (1, 1039, 264, 1),
    "split_padded_merged_odd": (1, 2116, 136, 4),
    "split_full_merged_pairs": (1, 16437, 32, 16),
    "wg_padded_1_s": (1, 1, 3, 1),
    "wg_padded_2_s": (1, 5, 9, 1),
    "wg_padded_4_s": (1, 33, 33, 1),
    "wg_padded_8_s": (65, 66, 33, 1),
    "wg_padded_16_s": (65, 513, 9, 3),
    "wg_full_2_s": (1, 65, 1, 1),
    "wg_full_4_s": (1, 2049, 1, 1),
    "wg_full_8_s": (41, 69, 66, 66),
    "wg_full_16_s": (33, 156, 70, 70),
    "wg_full_16_s_f32": (38, 276, 33, 33),
    "wg_wide_1_s": (1, 1, 65, 1),
    "wg_wide_2_s": (1, 2, 65, 1),
    "wg_wide_4_s": (1, 3, 513, 1),
    "wg_wide_8_s": (1, 5, 514, 1),
    "wg_wide_16_s": (65, 9, 519, 1),
    "wave_full_1_s": (1027, 2, 1, 1),
    "wave_packed_s": (1024, 1, 1, 1),
    "wave_full_2_s": (1033, 67, 1, 1),
    "wave_padded_2_s": (1032, 9, 5, 1),
    "split_padded_s": (1, 66, 33, 1),
    "split_full_s": (1, 2049, 2, 1),
    "split_full_merged_s": (1, 16391, 4, 1),
    "split_wide_s": (1, 41, 102, 2),
    "split_wide_merged_s": (1, 257, 133, 1),
}

# forward alone: many vectors a thread, of which a backward keeps fewer
FORWARD = {
    "wg_padded_8": (70, 65, 264, 1),
    "wg_padded_8_quarters": (33, 257, 144, 4),
    "wg_padded_16": (66, 264, 136, 1),
    "wg_padded_16_odd": (66, 130, 264, 8),
    "wg_full_8": (64, 530, 64, 1),
    "wg_full_8_one_channel_groups": (40, 637, 72, 72),
    "wg_full_16": (64, 8229, 8, 1),
    "wg_full_16_fours": (38, 1250, 72, 18),
    "wg_wide_16": (35, 26, 4144, 2),
    "wg_wide_16_halves": (73, 18, 3000, 2),
}

# many samples for workgroups of their own, which loop over them in a backward where
# they are of few pixels: rows of one group (layer norm) and others that no wavefront holds
MANY = {
    "layer_rows": (3001, 1, 1024, 1),
    "layer_rows_768": (2500, 1, 768, 1),
    "layer_rows_widest": (2200, 1, 4096, 1),
    "layer_rows_two_tiles": (1200, 1, 4096, 2),
    "layer_rows_halves": (2300, 1, 1000, 2),
    "layer_rows_s": (2600, 1, 515, 1),
    "two_pixels": (1103, 2, 1024, 1),
    "two_pixels_halves": (1301, 2, 1000, 2),
    "two_pixels_s": (1203, 2, 515, 1),
    "three_pixels_halves": (701, 3, 2056, 2),
    "four_pixels_full": (1501, 4, 512, 1),
    "four_pixels_padded": (1401, 4, 264, 1),
    "four_pixels_padded_halves": (1402, 4, 264, 2),
    "four_pixels_widest": (601, 4, 4096, 1),
    "few_pixels": (10000, 20, 64, 8),
    "few_pixels_fours": (2600, 20, 64, 16),
    "few_pixels_padded": (2500, 20, 40, 1),
    "few_pixels_padded_odd": (2401, 20, 40, 4),
    "few_pixels_s": (2500, 70, 9, 3),
    "few_pixels_one_channel_groups_s": (2100, 200, 3, 3),
}

COMBOS = [("silu", 0.2), ("relu", 0.0), ("none", 0.3), ("silu", 0.0)]
GRADIENTS = {"bf16": [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")], "f32": [("f32", "f32")]}


def combos(k):
    """Activation and dropout of the k-th shape's runs: one with, one without SiLU."""
    return [COMBOS[k % 2 * 3], COMBOS[1 + k % 2]]
