// How deep the list of a segment goes (sample.hip): plain arithmetic, which the host's tests call too.
#pragma once

namespace sf {

// of every (row, segment): a histogram of bins, from the bucket of the segment's largest downward, and a list of tokens
constexpr int SAMPLE_BINS = 256, SAMPLE_ROOM = 512;

// Bins that have counted all that lies in them.  bounded: nothing below `bound` was counted; then the last bin, which stands for
// all that lies below it too, never has, however far below the largest the bound is.
constexpr int sample_whole_bins(bool bounded, int top_bucket, int bound_bucket) {
  if (!bounded) return SAMPLE_BINS;
  return top_bucket - bound_bucket < SAMPLE_BINS - 1 ? top_bucket - bound_bucket : SAMPLE_BINS - 1;
}

// Whether the list may take a bin of cnt elements: upto lie in it and above it; none is taken once the segment alone has k.
constexpr bool sample_takes(int bin, int cnt, int upto, int whole_bins, int k) {
  return upto <= SAMPLE_ROOM && bin < whole_bins && upto - cnt < k;
}

}  // namespace sf
