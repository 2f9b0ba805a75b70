"""Sizes at which 4-bit products are compared with 64 bits besides those of mx4_sizes.py: what each stands for is checked by
test_mx4_launches.py. Groups are named by the rows of each."""
# tiles of every height, empty groups, groups of one row; 8 groups are looked up in another way than other numbers of them
EIGHT = (0, 160, 185, 224, 256, 700, 1075, 1100)
TWELVE = (0, 1, 33, 128, 160, 185, 224, 256, 257, 400, 700, 1356)
# groups, columns, elements of a row: more than two rounds of tiles, odd and even numbers of k-steps; the last round more and less
# than half full. One group: without offsets.
PERSISTENT = [(EIGHT, 16400, 544), (EIGHT, 16400, 1024), (TWELVE, 8720, 544), (TWELVE, 8720, 800),
              ((3000,), 16400, 544), ((3000,), 16400, 800)]
# a tile for each workgroup; reductions of 16384 and more cut their tiles otherwise
LARGE = [(EIGHT, 4112, 544), (EIGHT, 4112, 800), ((1000, 900, 1100), 4112, 544), ((1000, 900, 1100), 4112, 1024),
         ((1100,), 4112, 16384), ((1100,), 4112, 16416), ((700, 0, 1400), 4112, 16416)]
# the experts' FFN: groups, d_ff, d_model. d_ff = 128 modulo 256: rows of H that end in the middle of a run of scales
GATEUP_PERSISTENT = [(EIGHT, 4224, 512), (TWELVE, 4224, 1024), ((3000,), 8320, 512), (TWELVE, 4096, 1536)]
GATEUP_LARGE = [(EIGHT, 1408, 512), ((1000, 900, 1100), 2944, 1024), (EIGHT, 1408, 1536)]
GATEUP_ENDS = [((3, 14), 128, 512), ((10, 0, 30), 640, 1024), ((900, 600), 384, 512), ((1200, 1300), 640, 512)]      # smaller tiles
# Rows a multiple of 4 KB apart: n-tiles begin at k-steps of their own.
OWN_KSTEPS = [((1000,), 144, 8192), ((10, 0, 7, 20, 3, 1, 1, 35), 2064, 16384), ((1000,), 272, 8192), ((513,), 272, 16384),
              ((100, 30, 200, 60, 10, 0, 100, 200), 2064, 8192), ((1000,), 528, 8192), ((2100,), 272, 16384), ((1000,), 1040, 8192),
              ((700, 0, 1400), 528, 8192), ((1000,), 2064, 8192), ((700, 200, 1200), 1040, 16384)]
GATEUP_OWN_KSTEPS = [((5, 0, 12), 384, 8192), ((300, 213), 640, 8192), ((600, 0, 400), 640, 8192), ((60, 0, 150, 40) * 4, 1408, 8192),
                     ((16,) * 5, 256, 16384)]
# One matrix and three: where the NaN of a row and of a column have to stay.
NAN = [((77,), 4112, 2080), ((1000,), 2064, 96), ((513,), 4112, 2080), ((1000,), 8208, 544), ((3000,), 16400, 800),
       ((1000, 900, 1100), 4112, 544)]
